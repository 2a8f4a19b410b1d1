// The gated linear recurrence: its scan over a sequence, one step of it, and its backward pass.
// Part of libapms.so: included by layers.cu.
#pragma once

namespace {

// Per channel, with z = sigmoid(-gate) and a = 1 - z = sigmoid(gate):  h_t = a_t h_(t-1) + z_t x_t, computed as h + z (x - h), which keeps a state that
// has reached its input to the last bit however long it is held (a rounded a would forget 2^-24 of it every step).  A span of steps takes
// h to h + (B - C h): B what the span makes of h = 0, C = 1 - the product of its a, formed as C + z (1 - C) for the same reason.
// Backward, with G_t the gradient of h_t and k what arrives from later steps:  G = dh + k,  dx = z G,  dgate = G (h_(t-1) - x) a z,  k = a G.
//
// A warp takes 128 bytes of channels (a slab: 64 16-bit or 32 binary32 ones) and a span of kSpan steps, so that a span's operands fit into
// registers; kWarps warps lie one behind the other in time (in a short sequence fewer, and several slabs a CTA), and up to 16 CTAs of a
// cluster behind one another too, where there are too few channels to fill the GPU: a round of the loop is kSpan * warps * CTAs steps.  Per round each warp forms its
// span's (B, C); CTAs exchange the warps', clusters the CTAs' through one another's shared memory; then each warp runs its steps from its own first
// state.  The rounds' operands come by asynchronous copies, `kStages` rounds ahead, each warp its own: no barrier is needed for them.  Inputs are read once and outputs
// written once: bound by HBM.
constexpr int kSpan = 16, kWarps = 8, kScanThreads = kWarps * 32, kStages = 2;
constexpr int kRowBytes = 128, kSpanBytes = kSpan * kRowBytes;
constexpr int kMostCluster = 16, kMostClusterBack = 8;
constexpr int kStartsPad = 64;                                      // rows of starts: whole slabs of either type

struct ScanArgs {
    int64_t batch, steps, width;
    const void *x, *gate, *dh;
    int64_t x_batch, x_step, gate_batch, gate_step, dh_batch, dh_step;
    const float *state, *dlast;
    void *h, *dx, *dgate;
    float *last, *starts, *dstate;
    int64_t slabs, spans, starts_width;
    int warps, rounds;                                              // warps in time; rounds of the loop
    int pairs;                                                      // outputs can be written two 16-bit elements at a time
};

// A warp's channels: one a lane in binary32, two in 16 bits; values as pairs, the second unused in binary32.
template <int TYPE> constexpr int kLaneChannels = TYPE == APMS_GRAD_F32 ? 1 : 2;

__device__ __forceinline__ float exp2_fast(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float reciprocal_fast(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
constexpr float kLog2E = 1.44269504f;

// z = 1 / (1 + exp(gate)).  For 16-bit types by the approximate exponential and reciprocal (about 2^-21 relative to z at |gate| = 10, beside their
// 2^-9 and 2^-12); in binary32 by the library's.
template <int TYPE>
__device__ __forceinline__ float taken(float gate)
{
    if (TYPE == APMS_GRAD_F32) return 1.0f / (1.0f + expf(gate));
    return reciprocal_fast(1.0f + exp2_fast(gate * kLog2E));
}
// The smaller of z and a, with the sign of the gate: both come from it without cancellation.
template <int TYPE>
__device__ __forceinline__ float smaller(float gate)
{
    const float m = fabsf(gate);
    const float p = TYPE == APMS_GRAD_F32 ? expf(-m) / (1.0f + expf(-m)) : exp2_fast(-m * kLog2E) * reciprocal_fast(1.0f + exp2_fast(-m * kLog2E));
    return copysignf(p, gate);
}

__device__ __forceinline__ void copy_async16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy_async4(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

// `valid` rows of a slab to the warp's place in shared memory, 128 bytes apart.  UNIT: the bytes that rows are aligned to.
template <int TYPE, int UNIT>
__device__ __forceinline__ void fetch(uint32_t to, const void* rows, int64_t stride, int valid, int channels, int lane)
{
    constexpr int ES = kBytes<TYPE>;
    const char* p = static_cast<const char*>(rows);
    if constexpr (UNIT == 16) {
        const int piece = lane & 7;
#pragma unroll
        for (int r = lane >> 3; r < kSpan; r += 4)
            if (r < valid && piece * (16 / ES) < channels) copy_async16(to + r * kRowBytes + piece * 16, p + r * stride * ES + piece * 16);
    } else if constexpr (UNIT == 4) {
#pragma unroll
        for (int r = 0; r < kSpan; ++r)
            if (r < valid && lane * (4 / ES) < channels) copy_async4(to + r * kRowBytes + lane * 4, p + r * stride * ES + lane * 4);
    } else {
        const uint16_t* q = static_cast<const uint16_t*>(rows);
#pragma unroll
        for (int r = 0; r < kSpan; ++r) {
            if (r >= valid || lane * 2 >= channels) break;
            const uint32_t a = q[r * stride + lane * 2], b = lane * 2 + 1 < channels ? q[r * stride + lane * 2 + 1] : 0u;
            asm volatile("st.shared.u32 [%0], %1;" :: "r"(to + r * kRowBytes + lane * 4), "r"(a | b << 16) : "memory");
        }
    }
}

__device__ __forceinline__ uint32_t shared_word(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
template <int TYPE>
__device__ __forceinline__ float2 pair_at(uint32_t a)
{
    const uint32_t w = shared_word(a);
    if constexpr (TYPE == APMS_GRAD_F32) return make_float2(__uint_as_float(w), 0.0f);
    else return unpack16<TYPE>(w);
}

// One arithmetic operation on a lane's channels.
template <int TYPE> __device__ __forceinline__ float2 fma_(float2 a, float2 b, float2 c)
{
    if constexpr (TYPE == APMS_GRAD_F32) return make_float2(fmaf(a.x, b.x, c.x), 0.0f);
    else return fma2(a, b, c);
}
template <int TYPE> __device__ __forceinline__ float2 add_(float2 a, float2 b)
{
    if constexpr (TYPE == APMS_GRAD_F32) return make_float2(a.x + b.x, 0.0f);
    else return add2(a, b);
}
template <int TYPE> __device__ __forceinline__ float2 sub_(float2 a, float2 b)
{
    if constexpr (TYPE == APMS_GRAD_F32) return make_float2(a.x - b.x, 0.0f);
    else return fma2(b, both(-1.0f), a);
}
template <int TYPE> __device__ __forceinline__ float2 mul_(float2 a, float2 b)
{
    if constexpr (TYPE == APMS_GRAD_F32) return make_float2(a.x * b.x, 0.0f);
    else return mul2(a, b);
}
__device__ __forceinline__ float2 minus(float2 a) { return make_float2(-a.x, -a.y); }

template <int TYPE>
__device__ __forceinline__ void store_pair(void* p, int64_t at, float2 v, int mine, bool pairs)
{
    if constexpr (TYPE == APMS_GRAD_F32) {
        static_cast<float*>(p)[at] = v.x;
    } else if (pairs) {
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p) + at) = pack16<TYPE>(v);
    } else {
        store1<TYPE>(p, at, v.x);
        if (mine > 1) store1<TYPE>(p, at + 1, v.y);
    }
}

// A span of steps as h -> B + (1 - C) h, for a lane's channels; in the backward pass k -> B + A k.
struct Span { float2 b, c; };

// Where a warp works: which sequence and slab, and what of a round.
template <int TYPE>
struct Place {
    int lane, warp, in_time, rank, ctas, mine, channels;           // mine: of this lane's channels, those that exist (0: none); channels: of the slab
    int64_t sequence, column;                                       // column: of the slab's first channel
    bool live;
    __device__ __forceinline__ explicit Place(const ScanArgs& a, int ctas_) : ctas(ctas_)
    {
        constexpr int WIDE = 32 * kLaneChannels<TYPE>;
        lane = threadIdx.x & 31; warp = threadIdx.x >> 5;
        in_time = warp & (a.warps - 1);
        rank = ctas > 1 ? (int)cluster_rank() : 0;
        const int64_t slab = (int64_t)(blockIdx.x / ctas) * (kWarps / a.warps) + warp / a.warps;
        live = slab < a.batch * a.slabs;
        sequence = live ? slab / a.slabs : 0;
        column = live ? (slab - sequence * a.slabs) * WIDE : 0;
        channels = live ? (int)min((int64_t)WIDE, a.width - column) : 0;
        mine = max(0, min(kLaneChannels<TYPE>, channels - lane * kLaneChannels<TYPE>));
    }
    // The span of this warp in a round, counted from the first step or, backward, from the last.
    __device__ __forceinline__ int64_t span(const ScanArgs& a, int round) const { return ((int64_t)round * ctas + rank) * a.warps + in_time; }
};

// Joins the warps' spans of a round: `first` becomes what this warp's span begins with, `carry` (of the round's beginning) that of the next round's.
// APPLY(span, state): the state behind a span; JOIN(earlier, later): both as one.
template <class Apply, class Join>
__device__ __forceinline__ void exchange(Span mine, float2& carry, float2& first, int round, int warps, int warp, int lane, int rank, int ctas,
                                         float4 (*spans)[kWarps][32], float4* of_ctas, Apply apply, Join join)
{
    float4 (*here)[32] = spans[ctas == 1 ? round & 1 : 0];        // a cluster's barrier keeps two rounds apart as well
    here[warp][lane] = make_float4(mine.b.x, mine.b.y, mine.c.x, mine.c.y);
    __syncthreads();
    const int base = warp & ~(warps - 1);
    auto at = [&](int w) { const float4 v = here[w][lane]; return Span{make_float2(v.x, v.y), make_float2(v.z, v.w)}; };
    if (ctas == 1) {
        float2 s = carry;
        for (int w = 0; w < warps; ++w) {
            if (base + w == warp) first = s;
            s = apply(at(base + w), s);
        }
        carry = s;
        return;
    }
    Span all = at(0), before = all;                                 // several CTAs: all their warps lie in time
    for (int w = 1; w < kWarps; ++w) {
        if (w == warp) before = all;
        all = join(all, at(w));
    }
    float4* slots = of_ctas + (round & 1) * ctas * 32;              // two rounds apart: a CTA is past its reading when it comes to the next round's barrier
    for (int r = warp; r < ctas; r += kWarps) {
        const uint32_t to = cluster_address(shared_address(slots + rank * 32 + lane), (uint32_t)r);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"(to), "f"(all.b.x), "f"(all.b.y), "f"(all.c.x), "f"(all.c.y) : "memory");
    }
    cluster_barrier();
    float2 s = carry;
    for (int r = 0; r < ctas; ++r) {
        if (r == rank) first = s;
        const float4 v = slots[r * 32 + lane];
        s = apply(Span{make_float2(v.x, v.y), make_float2(v.z, v.w)}, s);
    }
    carry = s;
    if (warp) first = apply(before, first);
}

// Shared memory: the ring, the warps' spans (twice, or once and the CTAs' twice).  Two CTAs fit an SM, backward with clusters of up to 8.
template <bool BACK> constexpr int kStageBytes = BACK ? 3 * kSpanBytes + 256 : 2 * kSpanBytes;
template <bool BACK>
constexpr size_t scan_shared(int ctas) { return (size_t)kStages * kWarps * kStageBytes<BACK> + (ctas == 1 ? 2 * kWarps : kWarps + 2 * ctas) * 32 * sizeof(float4); }

template <int TYPE, int UNIT>
__global__ void __launch_bounds__(kScanThreads, 2) k_scan(ScanArgs a, int ctas)
{
    extern __shared__ float4 room[];
    constexpr int LC = kLaneChannels<TYPE>;
    constexpr int STAGE = kStageBytes<false>;
    char* ring = reinterpret_cast<char*>(room);
    float4 (*spans)[kWarps][32] = reinterpret_cast<float4 (*)[kWarps][32]>(ring + kStages * kWarps * STAGE);
    float4* of_ctas = reinterpret_cast<float4*>(ring + kStages * kWarps * STAGE) + kWarps * 32;
    const Place<TYPE> me(a, ctas);
    const uint32_t my_ring = shared_address(ring) + me.warp * kStages * STAGE;
    const int64_t channel = me.column + me.lane * LC;
    const char* xs = static_cast<const char*>(a.x) + (me.sequence * a.x_batch + me.column) * kBytes<TYPE>;
    const char* gs = static_cast<const char*>(a.gate) + (me.sequence * a.gate_batch + me.column) * kBytes<TYPE>;

    auto steps_of = [&](int64_t span) { return me.live ? (int)max((int64_t)0, min((int64_t)kSpan, a.steps - span * kSpan)) : 0; };
    auto issue = [&](int round) {
        if (round < a.rounds) {
            const int64_t t = me.span(a, round) * kSpan;
            const int valid = steps_of(me.span(a, round));
            const uint32_t to = my_ring + (round % kStages) * STAGE;
            fetch<TYPE, UNIT>(to, xs + t * a.x_step * kBytes<TYPE>, a.x_step, valid, me.channels, me.lane);
            fetch<TYPE, UNIT>(to + kSpanBytes, gs + t * a.gate_step * kBytes<TYPE>, a.gate_step, valid, me.channels, me.lane);
        }
        copies_issued();
    };
    for (int r = 0; r < kStages; ++r) issue(r);
    if (ctas > 1) cluster_barrier();                                // every CTA has begun: its shared memory may be written

    float2 carry = make_float2(0.0f, 0.0f);
    const int64_t state_at = me.sequence * a.width + channel;
    if (a.state && me.mine > 0) {
        carry.x = a.state[state_at];
        if (me.mine > 1) carry.y = a.state[state_at + 1];
    }
    for (int round = 0; round < a.rounds; ++round) {
        const int64_t span = me.span(a, round);
        const int valid = steps_of(span);
        const uint32_t from = my_ring + (round % kStages) * STAGE + me.lane * 4;
        copies_done<kStages - 1>();
        __syncwarp();
        float2 x[kSpan], z[kSpan];
        Span mine = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
        for (int s = 0; s < kSpan; ++s) {
            x[s] = pair_at<TYPE>(from + s * kRowBytes);
            const float2 g = pair_at<TYPE>(from + kSpanBytes + s * kRowBytes);
            z[s].x = taken<TYPE>(g.x);
            z[s].y = LC > 1 ? taken<TYPE>(g.y) : 0.0f;
        }
        if (valid < kSpan) {                                        // behind the sequence the state stays
#pragma unroll
            for (int s = 0; s < kSpan; ++s)
                if (s >= valid) x[s] = z[s] = make_float2(0.0f, 0.0f);
        }
#pragma unroll
        for (int s = 0; s < kSpan; ++s) {
            mine.b = fma_<TYPE>(z[s], sub_<TYPE>(x[s], mine.b), mine.b);
            mine.c = fma_<TYPE>(z[s], sub_<TYPE>(both(1.0f), mine.c), mine.c);
        }
        __syncwarp();                                               // all lanes have read the stage
        issue(round + kStages);
        float2 h;
        exchange(mine, carry, h, round, a.warps, me.warp, me.lane, me.rank, ctas, spans, of_ctas,
                 [](const Span& s, float2 v) { return add_<TYPE>(v, fma_<TYPE>(minus(s.c), v, s.b)); },
                 [](const Span& e, const Span& l) {
                     return Span{add_<TYPE>(e.b, fma_<TYPE>(minus(l.c), e.b, l.b)), fma_<TYPE>(l.c, sub_<TYPE>(both(1.0f), e.c), e.c)};
                 });
        if (valid && me.mine) {
            if (a.starts) {
                float* start = a.starts + (me.sequence * a.spans + span) * a.starts_width + channel;
                start[0] = h.x;
                if (LC > 1) start[1] = h.y;
            }
            const int64_t first = (me.sequence * a.steps + span * kSpan) * a.width + channel;
#pragma unroll
            for (int s = 0; s < kSpan; ++s) {
                if (s >= valid) break;
                h = fma_<TYPE>(z[s], sub_<TYPE>(x[s], h), h);
                store_pair<TYPE>(a.h, first + s * a.width, h, me.mine, a.pairs);
            }
        }
    }
    if (me.rank == 0 && me.in_time == 0 && me.mine > 0 && a.last) {
        a.last[state_at] = carry.x;
        if (me.mine > 1) a.last[state_at + 1] = carry.y;
    }
}

template <int TYPE, int UNIT>
__global__ void __launch_bounds__(kScanThreads, 2) k_scan_back(ScanArgs a, int ctas)
{
    extern __shared__ float4 room[];
    constexpr int LC = kLaneChannels<TYPE>, STAGE = kStageBytes<true>;
    char* ring = reinterpret_cast<char*>(room);
    float4 (*spans)[kWarps][32] = reinterpret_cast<float4 (*)[kWarps][32]>(ring + kStages * kWarps * STAGE);
    float4* of_ctas = reinterpret_cast<float4*>(ring + kStages * kWarps * STAGE) + kWarps * 32;
    const Place<TYPE> me(a, ctas);
    const uint32_t my_ring = shared_address(ring) + me.warp * kStages * STAGE;
    const int64_t channel = me.column + me.lane * LC;
    const char* xs = static_cast<const char*>(a.x) + (me.sequence * a.x_batch + me.column) * kBytes<TYPE>;
    const char* gs = static_cast<const char*>(a.gate) + (me.sequence * a.gate_batch + me.column) * kBytes<TYPE>;
    const char* ds = static_cast<const char*>(a.dh) + (me.sequence * a.dh_batch + me.column) * kBytes<TYPE>;
    const float* starts = a.starts + me.sequence * a.spans * a.starts_width + channel;

    // Rounds go backward in time: span counts from the last one.
    auto span_of = [&](int round) { return a.spans - 1 - me.span(a, round); };
    auto steps_of = [&](int64_t span) { return me.live && span >= 0 ? (int)min((int64_t)kSpan, a.steps - span * kSpan) : 0; };
    auto issue = [&](int round) {
        if (round < a.rounds) {
            const int64_t span = span_of(round), t = span * kSpan;
            const int valid = steps_of(span);
            const uint32_t to = my_ring + (round % kStages) * STAGE;
            fetch<TYPE, UNIT>(to, xs + t * a.x_step * kBytes<TYPE>, a.x_step, valid, me.channels, me.lane);
            fetch<TYPE, UNIT>(to + kSpanBytes, gs + t * a.gate_step * kBytes<TYPE>, a.gate_step, valid, me.channels, me.lane);
            fetch<TYPE, UNIT>(to + 2 * kSpanBytes, ds + t * a.dh_step * kBytes<TYPE>, a.dh_step, valid, me.channels, me.lane);
            if (valid) {                                            // rows of starts hold whole slabs
                const float* start = starts + span * a.starts_width;
                copy_async4(to + 3 * kSpanBytes + me.lane * LC * 4, start);
                if (LC > 1) copy_async4(to + 3 * kSpanBytes + me.lane * 8 + 4, start + 1);
            }
        }
        copies_issued();
    };
    for (int r = 0; r < kStages; ++r) issue(r);
    if (ctas > 1) cluster_barrier();                                // every CTA has begun: its shared memory may be written

    float2 carry = make_float2(0.0f, 0.0f);
    const int64_t state_at = me.sequence * a.width + channel;
    if (a.dlast && me.mine > 0) {
        carry.x = a.dlast[state_at];
        if (me.mine > 1) carry.y = a.dlast[state_at + 1];
    }
    for (int round = 0; round < a.rounds; ++round) {
        const int64_t span = span_of(round);
        const int valid = steps_of(span);
        const uint32_t stage = my_ring + (round % kStages) * STAGE, from = stage + me.lane * 4;
        copies_done<kStages - 1>();
        __syncwarp();
        float2 p[kSpan];                                            // the smaller of z and a, with the gate's sign
#pragma unroll
        for (int s = 0; s < kSpan; ++s) {
            const float2 g = pair_at<TYPE>(from + kSpanBytes + s * kRowBytes);
            p[s].x = smaller<TYPE>(g.x);
            p[s].y = LC > 1 ? smaller<TYPE>(g.y) : 0.0f;
        }
        auto z_of = [](float2 v) {
            return make_float2(__float_as_int(v.x) < 0 ? 1.0f + v.x : v.x, LC > 1 ? (__float_as_int(v.y) < 0 ? 1.0f + v.y : v.y) : 0.0f);
        };
        Span mine = {make_float2(0.0f, 0.0f), both(1.0f)};
#pragma unroll
        for (int s = kSpan - 1; s >= 0; --s) {
            if (s >= valid) continue;
            const float2 g = add_<TYPE>(pair_at<TYPE>(from + 2 * kSpanBytes + s * kRowBytes), mine.b), nz = minus(z_of(p[s]));
            mine.b = fma_<TYPE>(nz, g, g);
            mine.c = fma_<TYPE>(nz, mine.c, mine.c);
        }
        float2 k;
        exchange(mine, carry, k, round, a.warps, me.warp, me.lane, me.rank, ctas, spans, of_ctas,
                 [](const Span& s, float2 v) { return fma_<TYPE>(s.c, v, s.b); },
                 [](const Span& e, const Span& l) { return Span{fma_<TYPE>(l.c, e.b, l.b), mul_<TYPE>(l.c, e.c)}; });
        if (valid && me.mine) {
            float2 h = LC > 1 ? make_float2(__uint_as_float(shared_word(stage + 3 * kSpanBytes + me.lane * 8)), __uint_as_float(shared_word(stage + 3 * kSpanBytes + me.lane * 8 + 4)))
                              : make_float2(__uint_as_float(shared_word(stage + 3 * kSpanBytes + me.lane * 4)), 0.0f);
            float2 d[kSpan];                                        // h_(t-1) - x_t
#pragma unroll
            for (int s = 0; s < kSpan; ++s) {
                d[s] = sub_<TYPE>(h, pair_at<TYPE>(from + s * kRowBytes));
                h = fma_<TYPE>(minus(z_of(p[s])), d[s], h);
            }
            const int64_t first = (me.sequence * a.steps + span * kSpan) * a.width + channel;
#pragma unroll
            for (int s = kSpan - 1; s >= 0; --s) {
                if (s >= valid) continue;
                const float2 g = add_<TYPE>(pair_at<TYPE>(from + 2 * kSpanBytes + s * kRowBytes), k), z = z_of(p[s]);
                const float2 q = make_float2(fabsf(p[s].x), fabsf(p[s].y)), az = fma_<TYPE>(minus(q), q, q);
                store_pair<TYPE>(a.dx, first + s * a.width, mul_<TYPE>(z, g), me.mine, a.pairs);
                store_pair<TYPE>(a.dgate, first + s * a.width, mul_<TYPE>(mul_<TYPE>(g, d[s]), az), me.mine, a.pairs);
                k = fma_<TYPE>(minus(z), g, g);
            }
        }
        __syncwarp();                                               // all lanes have read the stage
        issue(round + kStages);
    }
    if (me.rank == 0 && me.in_time == 0 && me.mine > 0 && a.dstate) {
        a.dstate[state_at] = carry.x;
        if (me.mine > 1) a.dstate[state_at + 1] = carry.y;
    }
}

// ------------------------------------------------------------------------------------------ one step

struct StepArgs {
    int64_t batch, width, x_stride, gate_stride;
    const void *x, *gate;
    const float* state;
    void* h;
    float* next;
};

// One token of each sequence against its state: eight channels a thread.  Latency: one launch.
template <int TYPE>
__global__ void __launch_bounds__(128) k_scan_step(StepArgs a)
{
    const int64_t u = (int64_t)blockIdx.x * 128 + threadIdx.x, per_row = a.width / 8;
    if (u >= a.batch * per_row) return;
    const int64_t row = u / per_row, col = (u - row * per_row) * 8;
    float x[8], g[8], h[8];
    const Eight<TYPE> xr = load8<TYPE>(a.x, row * a.x_stride + col), gr = load8<TYPE>(a.gate, row * a.gate_stride + col);
    const Eight<APMS_GRAD_F32> hr = load8<APMS_GRAD_F32>(a.state, u * 8);
    values8<TYPE>(x, xr);
    values8<TYPE>(g, gr);
    values8<APMS_GRAD_F32>(h, hr);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = fmaf(taken<TYPE>(g[j]), x[j] - h[j], h[j]);
    store8<APMS_GRAD_F32>(a.next, u * 8, h);
    store8<TYPE>(a.h, u * 8, h);
}

template <int TYPE>
__global__ void __launch_bounds__(128) k_scan_step_any(StepArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (i >= a.batch * a.width) return;
    const int64_t row = i / a.width, col = i - row * a.width;
    const float before = a.state[i], h = fmaf(taken<TYPE>(load1<TYPE>(a.gate, row * a.gate_stride + col)), load1<TYPE>(a.x, row * a.x_stride + col) - before, before);
    a.next[i] = h;
    store1<TYPE>(a.h, i, h);
}

// ------------------------------------------------------------------------------------------ host

// Warps in time: as many as the sequence has spans, up to 8.  CTAs in time: while there are fewer than two for each of about 148 SMs, and a round has
// something for each.  Both by the sizes alone, so that results are the same on every GPU.
int plan_scan(ScanArgs& a, int type, int most)
{
    const int64_t wide = type == APMS_GRAD_F32 ? 32 : 64;
    a.slabs = (a.width + wide - 1) / wide;
    a.spans = (a.steps + kSpan - 1) / kSpan;
    a.starts_width = (a.width + kStartsPad - 1) / kStartsPad * kStartsPad;
    a.warps = 1;
    while (a.warps < kWarps && a.warps < a.spans) a.warps *= 2;
    int ctas = 1;
    while (ctas < most && a.batch * a.slabs * ctas * 2 <= 296 && (int64_t)ctas * 2 * kWarps <= a.spans) ctas *= 2;
    a.rounds = (int)((a.spans + (int64_t)a.warps * ctas - 1) / ((int64_t)a.warps * ctas));
    return ctas;
}

bool rows_on(const void* p, int64_t batch, int64_t batch_stride, int64_t steps, int64_t step_stride, int64_t es, int64_t unit)
{
    return (uintptr_t)p % unit == 0 && (batch <= 1 || batch_stride * es % unit == 0) && (steps <= 1 || step_stride * es % unit == 0);
}

template <int TYPE, int UNIT, bool BACK>
cudaError_t launch_scan_unit(const ScanArgs& a, int ctas, cudaStream_t stream)
{
    auto kernel = BACK ? k_scan_back<TYPE, UNIT> : k_scan<TYPE, UNIT>;
    static Raised raised[kMostDevices];
    cudaError_t e = raise_limits(raised, reinterpret_cast<const void*>(kernel), scan_shared<BACK>(BACK ? kMostClusterBack : kMostCluster), true);
    if (e != cudaSuccess) return e;
    const int64_t per_cta = kWarps / a.warps, clusters = (a.batch * a.slabs + per_cta - 1) / per_cta;
    if (clusters * ctas > 0x7fffffff) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)(clusters * ctas));
    if (ctas == 1) return launch(kernel, grid, kScanThreads, scan_shared<BACK>(1), stream, false, a, ctas);
    return launch_clusters(kernel, ctas, grid, kScanThreads, scan_shared<BACK>(ctas), stream, a, ctas);
}

template <int TYPE, bool BACK>
cudaError_t launch_scan(const ScanArgs& a, int ctas, cudaStream_t stream)
{
    constexpr int64_t ES = kBytes<TYPE>;
    auto on = [&](int64_t unit) {
        return a.width * ES % unit == 0 && rows_on(a.x, a.batch, a.x_batch, a.steps, a.x_step, ES, unit) && rows_on(a.gate, a.batch, a.gate_batch, a.steps, a.gate_step, ES, unit) &&
               (!BACK || rows_on(a.dh, a.batch, a.dh_batch, a.steps, a.dh_step, ES, unit));
    };
    if (on(16)) return launch_scan_unit<TYPE, 16, BACK>(a, ctas, stream);
    if (ES == 4 || on(4)) return launch_scan_unit<TYPE, 4, BACK>(a, ctas, stream);
    if constexpr (ES == 2) return launch_scan_unit<TYPE, 2, BACK>(a, ctas, stream);
    return cudaErrorInvalidValue;
}

template <bool BACK>
cudaError_t launch_scan_types(const ScanArgs& a, int type, int ctas, cudaStream_t stream)
{
    return type == APMS_GRAD_F32 ? launch_scan<APMS_GRAD_F32, BACK>(a, ctas, stream)
         : type == APMS_GRAD_BF16 ? launch_scan<APMS_GRAD_BF16, BACK>(a, ctas, stream) : launch_scan<APMS_GRAD_F16, BACK>(a, ctas, stream);
}

template <int TYPE>
cudaError_t launch_step(const StepArgs& a, bool vector, cudaStream_t stream)
{
    const int64_t n = vector ? a.batch * a.width / 8 : a.batch * a.width;
    return launch(vector ? k_scan_step<TYPE> : k_scan_step_any<TYPE>, dim3((unsigned)((n + 127) / 128)), 128, 0, stream, false, a);
}

constexpr int64_t kMostScan = (int64_t)1 << 31, kMostScanElements = (int64_t)1 << 40;

bool scan_sizes(int64_t batch, int64_t steps, int64_t width)
{
    return batch >= 0 && steps >= 0 && width >= 1 && batch < kMostScan && steps < kMostScan && width < kMostScan && batch * width <= kMostScan && batch * width * steps <= kMostScanElements;
}

apms_status scan_check(const char* who, int64_t batch, int64_t steps, int64_t width, apms_grad_type type)
{
    if (!scan_sizes(batch, steps, width))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld sequences of %lld steps of %lld channels: needs none below 0, width >= 1, batch * width <= 2^31 and at most 2^40 elements", who,
                             (long long)batch, (long long)steps, (long long)width);
    if (!known_type(type)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: unknown element type", who);
    return APMS_OK;
}

}  // namespace

extern "C" {

size_t apms_gated_scan_starts_bytes(int64_t batch, int64_t steps, int64_t width)
{
    if (!scan_sizes(batch, steps, width)) return 0;
    return (size_t)batch * (size_t)((steps + kSpan - 1) / kSpan) * (size_t)((width + kStartsPad - 1) / kStartsPad * kStartsPad) * sizeof(float);
}

apms_status apms_gated_scan(const apms_gated_scan_args* args, void* cuda_stream)
{
    const char* who = "apms_gated_scan";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_gated_scan_args& g = *args;
    const apms_status st = scan_check(who, g.batch, g.steps, g.width, g.type);
    if (st != APMS_OK) return st;
    if (g.batch == 0) return APMS_OK;
    if (!g.last || (g.steps && (!g.x || !g.gate || !g.h))) return operator_fail(APMS_ERR_INVALID_ARG, "%s: x, gate, h or last is NULL", who);
    if (g.x_batch_stride < 0 || g.x_step_stride < 0 || g.gate_batch_stride < 0 || g.gate_step_stride < 0) return operator_fail(APMS_ERR_INVALID_ARG, "%s: a stride is below 0", who);
    if (!on_element(g.x, g.type) || !on_element(g.gate, g.type) || !on_element(g.h, g.type) || !on_element(g.state, APMS_GRAD_F32) || !on_element(g.last, APMS_GRAD_F32) || !on_element(g.starts, APMS_GRAD_F32))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    ScanArgs a = {};
    a.batch = g.batch; a.steps = g.steps; a.width = g.width;
    a.x = g.x; a.x_batch = g.x_batch_stride; a.x_step = g.x_step_stride;
    a.gate = g.gate; a.gate_batch = g.gate_batch_stride; a.gate_step = g.gate_step_stride;
    a.state = g.state; a.h = g.h; a.last = g.last; a.starts = g.starts;
    const int ctas = plan_scan(a, g.type, kMostCluster);
    a.pairs = a.width % 2 == 0 && (uintptr_t)a.h % 4 == 0;
    OPERATOR_CUDA("apms_gated_scan", launch_scan_types<false>(a, g.type, ctas, (cudaStream_t)cuda_stream));
    return APMS_OK;
}

apms_status apms_gated_scan_backward(const apms_gated_scan_backward_args* args, void* cuda_stream)
{
    const char* who = "apms_gated_scan_backward";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_gated_scan_backward_args& g = *args;
    const apms_status st = scan_check(who, g.batch, g.steps, g.width, g.type);
    if (st != APMS_OK) return st;
    if (g.batch == 0) return APMS_OK;
    if (g.steps && (!g.dh || !g.x || !g.gate || !g.starts || !g.dx || !g.dgate)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: dh, x, gate, starts, dx or dgate is NULL", who);
    if (g.x_batch_stride < 0 || g.x_step_stride < 0 || g.gate_batch_stride < 0 || g.gate_step_stride < 0 || g.dh_batch_stride < 0 || g.dh_step_stride < 0)
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: a stride is below 0", who);
    if (!on_element(g.x, g.type) || !on_element(g.gate, g.type) || !on_element(g.dh, g.type) || !on_element(g.dx, g.type) || !on_element(g.dgate, g.type) ||
        !on_element(g.starts, APMS_GRAD_F32) || !on_element(g.dlast, APMS_GRAD_F32) || !on_element(g.dstate, APMS_GRAD_F32))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    ScanArgs a = {};
    a.batch = g.batch; a.steps = g.steps; a.width = g.width;
    a.x = g.x; a.x_batch = g.x_batch_stride; a.x_step = g.x_step_stride;
    a.gate = g.gate; a.gate_batch = g.gate_batch_stride; a.gate_step = g.gate_step_stride;
    a.dh = g.dh; a.dh_batch = g.dh_batch_stride; a.dh_step = g.dh_step_stride;
    a.starts = const_cast<float*>(g.starts); a.dlast = g.dlast; a.dx = g.dx; a.dgate = g.dgate; a.dstate = g.dstate;
    const int ctas = plan_scan(a, g.type, kMostClusterBack);
    a.pairs = a.width % 2 == 0 && (uintptr_t)a.dx % 4 == 0 && (uintptr_t)a.dgate % 4 == 0;
    OPERATOR_CUDA("apms_gated_scan_backward", launch_scan_types<true>(a, g.type, ctas, (cudaStream_t)cuda_stream));
    return APMS_OK;
}

apms_status apms_gated_scan_step(const apms_gated_scan_step_args* args, void* cuda_stream)
{
    const char* who = "apms_gated_scan_step";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_gated_scan_step_args& g = *args;
    const apms_status st = scan_check(who, g.batch, 1, g.width, g.type);
    if (st != APMS_OK) return st;
    if (g.batch == 0) return APMS_OK;
    if (!g.x || !g.gate || !g.state || !g.next || !g.h) return operator_fail(APMS_ERR_INVALID_ARG, "%s: x, gate, state, next or h is NULL", who);
    if (g.x_stride < 0 || g.gate_stride < 0) return operator_fail(APMS_ERR_INVALID_ARG, "%s: a stride is below 0", who);
    if (!on_element(g.x, g.type) || !on_element(g.gate, g.type) || !on_element(g.h, g.type) || !on_element(g.state, APMS_GRAD_F32) || !on_element(g.next, APMS_GRAD_F32))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    const StepArgs a = {g.batch, g.width, g.x_stride, g.gate_stride, g.x, g.gate, g.state, g.h, g.next};
    const bool vector = rows_of_eight(a.x, a.batch, a.x_stride, a.width, g.type) && rows_of_eight(a.gate, a.batch, a.gate_stride, a.width, g.type) && on_16(a.h) && on_16(a.state) && on_16(a.next);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    OPERATOR_CUDA("apms_gated_scan_step", g.type == APMS_GRAD_F32 ? launch_step<APMS_GRAD_F32>(a, vector, stream)
                                        : g.type == APMS_GRAD_BF16 ? launch_step<APMS_GRAD_BF16>(a, vector, stream) : launch_step<APMS_GRAD_F16>(a, vector, stream));
    return APMS_OK;
}

}  // extern "C"
