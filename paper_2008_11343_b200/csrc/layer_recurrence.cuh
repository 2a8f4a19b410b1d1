// The gated linear recurrence: its scan over a sequence, one step of it, and its backward pass.
// Part of libapms.so: included by layers.cu.
#pragma once

namespace {

// Per channel, with z = sigmoid(-gate) and a = 1 - z = sigmoid(gate):  h_t = a_t h_(t-1) + z_t x_t, so within a span of 8 steps: one dependent operation a step (h + z (x - h) has
// two).  From span to span, with B what the span makes of h = 0, A the product of its a and C = 1 - A, formed as a C + z, a state goes to h + (B - C h) where the span keeps half of it or
// more: what the rounding of a, 2^-25, forgets of a state every step so adds up over a span at most, and a state that has reached its input stays there however long it is held.  Where
// the span forgets more than half, h + (B - C h) would leave the rounding of a state that is gone (2^-24 of it) in the one that is there; the state goes to B + A h.
// Backward, with G_t the gradient of h_t and k what arrives from later steps:  G = dh + k,  dx = z G,  dgate = G (h_(t-1) - x) a z,  k = G - z G;  a span takes k to
// B + A k.  A z below 2^-25 is lost there, as in binary32 at large: a gradient held over 10^5 such steps is off by some 10^-3.  The states come from `starts`, those that the forward pass
// had before every 8 steps, and x and gate again, h - z h + z x: h - z (h - x) would leave the rounding of a state that is gone, too.
//
// A lane holds 8 bytes of channels (two pairs of 16-bit ones, one pair of binary32), a warp a slab of 256 bytes, over a span of 8 steps, whose operands fit into registers.
// Eight warps lie one behind the other in time (in a short sequence fewer, and several slabs together): a round of the loop.  Per round each warp forms its span's (B, A or C),
// the first one takes the state through them, and each runs its steps from its own first state.  An SM holds two such teams: two CTAs, or, where there are too few slabs
// for that, the two halves of one CTA that take turns at a slab's rounds; one team forms its spans (bound by the exponentials and reciprocals) while the other one finishes.
// Where there are fewer slabs than SMs, a sequence is cut into segments, whose (B, A or C) a kernel of its own forms first; each segment then begins with the state behind those
// before it.  The operands come by asynchronous copies two rounds ahead, each warp its own.  Inputs are read once (before the last segment twice) and outputs written once.
// 8 x 4096 x 2048 bfloat16: 69 us on the same inputs again, 73 to 76 on new ones, 5.3 TB/s (in step, 16 warps: 86; clusters of two CTAs: 92; two channels a lane: 82); backward 119, and
// 127 to 132; 1 x 32,768 x 1024: 64 to 68 us (clusters of 16 CTAs that exchange every round: 135), backward 85.  With h + (B - C h) alone, and the states of the backward pass by
// h - z (h - x): 69, 116, 62 and 84.  Bound by HBM where there are slabs for two teams an SM; else by the rounds, whose exponentials and reciprocals take a quarter to a half of the time.
constexpr int kSpan = 8, kTeam = 8;                                 // steps; warps
constexpr int kRowBytes = 256;
constexpr int kStartsPad = 128;                                     // rows of starts: whole slabs of either type
constexpr int kStages = 2;

struct Rows { const void* p; int64_t batch, step; };                // bytes between sequences and steps
struct ScanArgs {
    int64_t batch, width;
    Rows x, gate, dh;
    const float *state, *dlast;
    void *h, *dx, *dgate;
    float *last, *starts, *dstate;
    float4* segments;                                               // what the segments' pieces do to a state: [sequence and slab][segment][piece][pair][lane]
    int64_t slabs, starts_width;
    int steps, spans, warps, parts, part_steps, pieces;             // warps in time of a team; segments, their steps, and the pieces that these are formed in
    int whole;                                                      // outputs can be written eight bytes at a time
};

template <int TYPE> constexpr int kPairs = TYPE == APMS_GRAD_F32 ? 1 : 2;
template <int TYPE> constexpr int kLaneChannels = 2 * kPairs<TYPE>;

__device__ __forceinline__ float exp2_fast(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float reciprocal_fast(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float lower(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float higher(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
constexpr float kLog2E = 1.44269504f, kLog2ELow = 1.92596303e-8f, kLn2 = 0.693147181f;               // log2(e) as a sum of two

// exp(gate) for z = 1 / (1 + exp(gate)), from the approximate power of two (2^-22).  In 16 bits the rounding of its argument adds about 2^-19 at |gate| = 16, beside the types' own
// 2^-9 and 2^-12; binary32 takes what was rounded off as a factor 1 + ln 2 * rest.  BOUND: finite for any gate.
template <int TYPE, bool BOUND>
__device__ __forceinline__ float2 exp_of(float2 gate)
{
    if constexpr (TYPE == APMS_GRAD_F32) {
        gate = make_float2(higher(lower(gate.x, 88.0f), -120.0f), higher(lower(gate.y, 88.0f), -120.0f));
        const float2 t = mul2(gate, both(kLog2E)), rest = fma2(gate, both(kLog2ELow), fma2(gate, both(kLog2E), make_float2(-t.x, -t.y)));
        const float2 e = make_float2(exp2_fast(t.x), exp2_fast(t.y));
        return fma2(mul2(rest, both(kLn2)), e, e);
    } else {
        float2 t = mul2(gate, both(kLog2E));
        if (BOUND) t = make_float2(lower(t.x, 127.0f), lower(t.y, 127.0f));
        return make_float2(exp2_fast(t.x), exp2_fast(t.y));
    }
}
// z and, for the backward pass, -z and a z.  Neither loses digits where z or a is small; a z below 2^-126 counts as 0.
template <int TYPE>
__device__ __forceinline__ float2 taken(float2 gate)
{
    const float2 d = add2(exp_of<TYPE, false>(gate), both(1.0f));
    return make_float2(reciprocal_fast(d.x), reciprocal_fast(d.y));
}
template <int TYPE>
__device__ __forceinline__ void minus_taken_and_slope(float2 gate, float2& nz, float2& az)
{
    const float2 e = exp_of<TYPE, true>(gate), d = fma2(e, both(-1.0f), both(-1.0f));              // e is finite: e z z is 0 where z is
    nz = make_float2(reciprocal_fast(d.x), reciprocal_fast(d.y));
    az = mul2(mul2(e, nz), nz);
}
__device__ __forceinline__ float2 minus(float2 a) { return make_float2(-a.x, -a.y); }
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return fma2(b, both(-1.0f), a); }  // exact product: rounded as a difference

__device__ __forceinline__ void copy_async16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy_async4(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

__device__ __forceinline__ uint2 shared_words(uint32_t a) { uint2 v; asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t shared_word(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }

// What a warp fetches of one input: a span's rows of a slab a time, to shared memory.  UNIT: the bytes that rows are aligned to.  Rows of 16-bit elements that are
// aligned to nothing more are copied by the aligned words that hold them, and shifted where they are read (8 x 4096 x 1001: 132 us; by plain loads of the elements 259).
template <int UNIT> constexpr int kPitch = kRowBytes + (UNIT == 2 ? 8 : 0);
template <int UNIT> constexpr int kSpanBytes = kSpan * kPitch<UNIT>;
template <int TYPE, int UNIT>
struct Feed {
    const char* p;                                                  // this lane's share of the next span
    uint32_t low;                                                   // UNIT 2: address of the first row of the span that is read
    __device__ __forceinline__ Feed(const Rows& r, int64_t sequence, int64_t column, int first, int lane)
        : p(static_cast<const char*>(r.p) + sequence * r.batch + column * kBytes<TYPE> + first * r.step), low((uint32_t)(uintptr_t)p)
    {
        if (UNIT == 16) p += (lane >> 4) * r.step + (lane & 15) * 16;
    }
    __device__ __forceinline__ void fetch(uint32_t to, const Rows& r, int64_t round, int valid, int channels, int lane)
    {
        const char* q = p;
        if constexpr (UNIT == 16) {
            to += lane * 16;                                        // (lane >> 4) rows and (lane & 15) pieces
            if ((lane & 15) * (16 / kBytes<TYPE>) < channels) {
#pragma unroll
                for (int s = 0; s < kSpan; s += 2) {
                    if ((lane >> 4) + s < valid) copy_async16(to + s * kRowBytes, q);
                    q += 2 * r.step;
                }
            }
        } else {
            const int bytes = channels * kBytes<TYPE> - lane * 4;   // from this lane's first word on
#pragma unroll
            for (int s = 0; s < kSpan; ++s) {
                if (s >= valid) break;
                const int shift = UNIT == 2 ? (int)((uintptr_t)q & 2) : 0;
                const char* words = q - shift + lane * 4;
                const uint32_t at = to + s * kPitch<UNIT> + lane * 4;
                if (bytes + shift > 0) copy_async4(at, words);
                if (bytes + shift > kRowBytes / 2) copy_async4(at + kRowBytes / 2, words + kRowBytes / 2);
                if (UNIT == 2 && bytes + shift > kRowBytes) copy_async4(at + kRowBytes, words + kRowBytes);        // lane 0: the last element's word
                q += r.step;
            }
        }
        p += round;
    }
    // Lane `lane`'s words of row s; at: its place in the span's first row.
    __device__ __forceinline__ uint2 words(uint32_t at, int s, const Rows& r) const
    {
        const uint2 w = shared_words(at + s * kPitch<UNIT>);
        if constexpr (UNIT != 2) return w;
        const uint32_t next = shared_word(at + s * kPitch<UNIT> + 8), shift = ((low + (uint32_t)(s * r.step)) & 2) * 8;
        return make_uint2(__funnelshift_r(w.x, w.y, shift), __funnelshift_r(w.y, next, shift));
    }
    __device__ __forceinline__ void read(int64_t round) { low += (uint32_t)round; }                       // on to the next span
    static __device__ __forceinline__ void zero(uint32_t at, int s, int lane)
    {
        asm volatile("st.shared.v2.u32 [%0], {%1, %1};" :: "r"(at + s * kPitch<UNIT>), "r"(0) : "memory");
        if (UNIT == 2 && lane == 31) asm volatile("st.shared.u32 [%0], %1;" :: "r"(at + s * kPitch<UNIT> + 8), "r"(0) : "memory");
    }
};

template <int TYPE>
__device__ __forceinline__ float2 pair_of(uint2 w, int p)
{
    if constexpr (TYPE == APMS_GRAD_F32) return make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    else return unpack16<TYPE>(p ? w.y : w.x);
}

// A lane's channels, rounded; WHOLE: all exist and can be written at once.
template <int TYPE, bool WHOLE>
__device__ __forceinline__ void store_lane(char* p, const float2* v, int mine)
{
    if constexpr (WHOLE) {
        *reinterpret_cast<uint2*>(p) = TYPE == APMS_GRAD_F32 ? make_uint2(__float_as_uint(v[0].x), __float_as_uint(v[0].y)) : make_uint2(pack16<TYPE>(v[0]), pack16<TYPE>(v[kPairs<TYPE> - 1]));
    } else {
#pragma unroll
        for (int i = 0; i < kLaneChannels<TYPE>; ++i)
            if (i < mine) store1<TYPE>(p, i, i & 1 ? v[i / 2].y : v[i / 2].x);
    }
}

// Where a warp works: which sequence and slab, which segment.
template <int TYPE>
struct Place {
    int in_time, mine, channels, part;                              // mine: of this lane's channels, those that exist; channels: of the slab
    int64_t slab, sequence, column, state_at;                       // column: of the slab's first channel; state_at: this lane's first element of a state
    bool live;
    __device__ __forceinline__ Place(const ScanArgs& a, int warp)   // warp: of the team
    {
        constexpr int LC = kLaneChannels<TYPE>, WIDE = 32 * LC;
        const int lane = threadIdx.x & 31;
        in_time = warp & (a.warps - 1);
        part = blockIdx.y;
        slab = (int64_t)blockIdx.x * (kTeam / a.warps) + warp / a.warps;
        live = slab < a.batch * a.slabs;
        sequence = live ? slab / a.slabs : 0;
        column = live ? (slab - sequence * a.slabs) * WIDE : 0;
        channels = live ? (int)min((int64_t)WIDE, a.width - column) : 0;
        mine = max(0, min(LC, channels - lane * LC));
        state_at = sequence * a.width + column + lane * LC;
    }
    __device__ __forceinline__ void load_state(float2* v, const float* from) const
    {
#pragma unroll
        for (int p = 0; p < kPairs<TYPE>; ++p) {
            v[p].x = from && 2 * p < mine ? from[state_at + 2 * p] : 0.0f;
            v[p].y = from && 2 * p + 1 < mine ? from[state_at + 2 * p + 1] : 0.0f;
        }
    }
    __device__ __forceinline__ void store_state(float* to, const float2* v) const
    {
#pragma unroll
        for (int p = 0; p < kPairs<TYPE>; ++p) {
            if (2 * p < mine) to[state_at + 2 * p] = v[p].x;
            if (2 * p + 1 < mine) to[state_at + 2 * p + 1] = v[p].y;
        }
    }
    // Where what this slab's piece s does to a state lies.
    __device__ __forceinline__ float4* piece(const ScanArgs& a, int s) const { return a.segments + ((slab * a.parts * a.pieces + s) * kPairs<TYPE>) * 32 + (threadIdx.x & 31); }
};

// One pair of channels over a span, and what it does to a state.  Forward: to h + (b + c h) with c = -C, or to b + c h with c = A: the sign of c says which (-0 where all is held).
struct Span { float2 b, c; };
__device__ __forceinline__ Span span_of(const float4& v) { return {make_float2(v.x, v.y), make_float2(v.z, v.w)}; }
struct Forward {
    // What is added to b + c h: 1 or 0 times h.
    static __device__ __forceinline__ float held(float c) { return __float_as_int(c) < 0 ? 1.0f : 0.0f; }
    static __device__ __forceinline__ float2 apply(const Span& s, float2 h) { return fma2(make_float2(held(s.c.x), held(s.c.y)), h, fma2(s.c, h, s.b)); }
    // c of a span whose A and C are known, and of two spans.
    static __device__ __forceinline__ float2 choose(float2 product, float2 forgotten)
    {
        return make_float2(forgotten.x > 0.5f ? fabsf(product.x) : -forgotten.x, forgotten.y > 0.5f ? fabsf(product.y) : -forgotten.y);
    }
    static __device__ __forceinline__ float both_of(float e, float l)
    {
        if (held(e) == 0.0f || held(l) == 0.0f) return (held(e) + e) * (held(l) + l);
        const float c = fmaf(l, -e, -e) - l;
        return c > 0.5f ? 1.0f - c : -c;                            // exact: 1 / 2 to 1 from 1
    }
    static __device__ __forceinline__ Span join(const Span& e, const Span& l) { return {apply(l, e.b), make_float2(both_of(e.c.x, l.c.x), both_of(e.c.y, l.c.y))}; }
};
struct Backward {
    static __device__ __forceinline__ float2 apply(const Span& s, float2 k) { return fma2(s.c, k, s.b); }
    static __device__ __forceinline__ Span join(const Span& e, const Span& l) { return {fma2(l.c, e.b, l.b), mul2(l.c, e.c)}; }
};

// Barriers of a team's warps: the spans are there (all wait), the states are there (the warps that join them only arrive); and of two teams' first warps: the carried state is.
template <int THREADS> __device__ __forceinline__ void bar_arrive(int id) { asm volatile("bar.arrive %0, %1;" :: "r"(id), "n"(THREADS) : "memory"); }
template <int THREADS> __device__ __forceinline__ void bar_sync(int id) { asm volatile("bar.sync %0, %1;" :: "r"(id), "n"(THREADS) : "memory"); }
constexpr int kFormed = 1, kJoined = 3, kCarried = 5;               // + the team

// Takes the state through a round's spans.  here: [pair][warp][lane], a span's (b, c), which becomes (the state that it begins with, .), from the group's first warp on.
template <int TYPE, class Way>
__device__ __forceinline__ void join_spans(float2* carry, int warps, float4* here)
{
    constexpr int P = kPairs<TYPE>;
    if (warps == kTeam) {
#pragma unroll
        for (int w0 = 0; w0 < kTeam; w0 += 4) {                     // loads first: four spans at a time
            float4 v[4][P];
#pragma unroll
            for (int w = 0; w < 4 * P; ++w) v[w / P][w % P] = here[(w % P * kTeam + w0 + w / P) * 32];
#pragma unroll
            for (int w = 0; w < 4 * P; ++w) {
                *reinterpret_cast<float2*>(here + (w % P * kTeam + w0 + w / P) * 32) = carry[w % P];
                carry[w % P] = Way::apply(span_of(v[w / P][w % P]), carry[w % P]);
            }
        }
    } else {
        for (int w = 0; w < warps; ++w)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const Span s = span_of(here[(p * kTeam + w) * 32]);
                *reinterpret_cast<float2*>(here + (p * kTeam + w) * 32) = carry[p];
                carry[p] = Way::apply(s, carry[p]);
            }
    }
}

// The state that a segment begins with: the first one through the `count` pieces before it, the first of which is `from`, the next ones `step` apart.
template <int TYPE, class Way>
__device__ __forceinline__ void through_pieces(float2* carry, const float4* from, int64_t step, int count)
{
    constexpr int P = kPairs<TYPE>;
    for (int s0 = 0; s0 < count; s0 += 4) {
        float4 v[4][P];
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (s0 + s < count) {
#pragma unroll
                for (int p = 0; p < P; ++p) v[s][p] = __ldcg(from + (s0 + s) * step + p * 32);
            }
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (s0 + s < count) {
#pragma unroll
                for (int p = 0; p < P; ++p) carry[p] = Way::apply(span_of(v[s][p]), carry[p]);
            }
    }
}

// One round's join by the team's first warps in time: with two teams the carried state comes from and goes to the other one's.
template <int TYPE, class Way, int TEAMS>
__device__ __forceinline__ void join_round(float2* carry, int round, int rounds, int warps, float4* here, float2* carried)
{
    constexpr int P = kPairs<TYPE>;
    const int lane = threadIdx.x & 31;
    if (TEAMS == 2 && round) {
        bar_sync<64>(kCarried + (round & 1));
#pragma unroll
        for (int p = 0; p < P; ++p) carry[p] = carried[p * 32 + lane];
    }
    join_spans<TYPE, Way>(carry, warps, here);
    if (TEAMS == 2 && round + 1 < rounds) {
#pragma unroll
        for (int p = 0; p < P; ++p) carried[p * 32 + lane] = carry[p];
        bar_arrive<64>(kCarried + (~round & 1));
    }
}

// A warp's span in, the state that it begins with out.
template <int TYPE>
__device__ __forceinline__ void put_span(const Span* mine, float4* at)
{
#pragma unroll
    for (int p = 0; p < kPairs<TYPE>; ++p) at[p * kTeam * 32] = make_float4(mine[p].b.x, mine[p].b.y, mine[p].c.x, mine[p].c.y);
}
template <int TYPE>
__device__ __forceinline__ void get_state(float2* state, const float4* at)
{
#pragma unroll
    for (int p = 0; p < kPairs<TYPE>; ++p) state[p] = *reinterpret_cast<const float2*>(at + p * kTeam * 32);
}

// Shared memory: the rings, the teams' spans, the carried state.
template <int UNIT, int TENSORS> constexpr int kStageBytes = TENSORS * kSpanBytes<UNIT>;
template <int UNIT, int TENSORS>
constexpr size_t scan_shared(int teams, int pairs) { return (size_t)teams * kTeam * kStages * kStageBytes<UNIT, TENSORS> + (size_t)pairs * 32 * (teams * kTeam * sizeof(float4) + sizeof(float2)); }

// What a span does to a state (also its A and C) from its gates and x, and a and z x of each step; VALID of its steps exist.
template <int TYPE, int UNIT, bool WHOLE>
__device__ __forceinline__ void form_span(Span* mine, float2* product, float2* forgotten, float2 (*keep)[kPairs<TYPE>], float2 (*zx)[kPairs<TYPE>], const Feed<TYPE, UNIT>& x_feed,
                                          const Feed<TYPE, UNIT>& gate_feed, const ScanArgs& a, uint32_t at, int valid)
{
    constexpr int P = kPairs<TYPE>;
#pragma unroll
    for (int p = 0; p < P; ++p) mine[p].b = forgotten[p] = both(0.0f);
#pragma unroll
    for (int s = 0; s < kSpan; ++s) {
        const uint2 g = gate_feed.words(at + kSpanBytes<UNIT>, s, a.gate), x = x_feed.words(at, s, a.x);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float2 z = taken<TYPE>(pair_of<TYPE>(g, p));
            keep[s][p] = sub2(both(1.0f), z);
            zx[s][p] = mul2(z, pair_of<TYPE>(x, p));
            if (!WHOLE && s >= valid) { keep[s][p] = both(1.0f); z = zx[s][p] = both(0.0f); }            // behind the sequence the state stays
            mine[p].b = fma2(keep[s][p], mine[p].b, zx[s][p]);
            forgotten[p] = fma2(keep[s][p], forgotten[p], z);
            product[p] = s ? mul2(product[p], keep[s][p]) : keep[s][p];
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) mine[p].c = Forward::choose(product[p], forgotten[p]);
}

template <int TYPE, int UNIT, int TEAMS>
__global__ void __launch_bounds__(TEAMS * kTeam * 32, 2 / TEAMS) k_scan(ScanArgs a)
{
    extern __shared__ float4 room[];
    constexpr int P = kPairs<TYPE>, LC = kLaneChannels<TYPE>, STAGE = kStageBytes<UNIT, 2>;
    const int warp = (threadIdx.x >> 5) % kTeam, team = threadIdx.x / (kTeam * 32), lane = threadIdx.x & 31;
    char* ring = reinterpret_cast<char*>(room);
    float4* here = reinterpret_cast<float4*>(ring + TEAMS * kTeam * kStages * STAGE);
    float2* carried = reinterpret_cast<float2*>(here + TEAMS * P * kTeam * 32);
    here += team * P * kTeam * 32 + warp * 32 + lane;
    const Place<TYPE> me(a, warp);
    const uint32_t my_ring = shared_address(ring) + (threadIdx.x >> 5) * kStages * STAGE;
    const int begin = me.part * a.part_steps, steps = me.live ? min(a.steps, begin + a.part_steps) : 0, round_steps = a.warps * kSpan;
    int t = begin + (team * a.warps + me.in_time) * kSpan, fetched = t;         // first step of the span that comes next, and of the one fetched next
    Feed<TYPE, UNIT> x_feed(a.x, me.sequence, me.column, t, lane), gate_feed(a.gate, me.sequence, me.column, t, lane);
    auto fetch = [&](uint32_t to) {
        x_feed.fetch(to, a.x, TEAMS * round_steps * a.x.step, steps - fetched, me.channels, lane);
        gate_feed.fetch(to + kSpanBytes<UNIT>, a.gate, TEAMS * round_steps * a.gate.step, steps - fetched, me.channels, lane);
        fetched += TEAMS * round_steps;
        copies_issued();
    };
#pragma unroll
    for (int r = 0; r < kStages; ++r) fetch(my_ring + r * STAGE);
    const int64_t row = a.width * kBytes<TYPE>;
    char* out = static_cast<char*>(a.h) + ((me.sequence * a.steps + t) * a.width + me.column + lane * LC) * kBytes<TYPE>;
    uint32_t stage = my_ring;
    float2 carry[P];                                                // in the first warps in time
    me.load_state(carry, a.state);
    if (me.part && me.in_time == 0 && team == 0) {
        wait_for_last_kernel();
        through_pieces<TYPE, Forward>(carry, me.piece(a, 0), P * 32, me.part * a.pieces);
    }
    const int rounds = (min(a.steps, begin + a.part_steps) - begin + round_steps - 1) / round_steps;
    for (int round = team; round < rounds; round += TEAMS) {
        const int valid = steps - t;                                // 8 or more: the whole span
        const uint32_t from = stage + lane * 8;
        copies_done<kStages - 1>();
        __syncwarp();
        float2 keep[kSpan][P], zx[kSpan][P], product[P], forgotten[P];
        Span mine[P];
        if (valid >= kSpan) form_span<TYPE, UNIT, true>(mine, product, forgotten, keep, zx, x_feed, gate_feed, a, from, valid);
        else form_span<TYPE, UNIT, false>(mine, product, forgotten, keep, zx, x_feed, gate_feed, a, from, valid);
        put_span<TYPE>(mine, here);
        bar_sync<kTeam * 32>(kFormed + team);
        if (me.in_time == 0) {
            join_round<TYPE, Forward, TEAMS>(carry, round, rounds, a.warps, here, carried);
            bar_arrive<kTeam * 32>(kJoined + team);
        }
        x_feed.read(TEAMS * round_steps * a.x.step);
        gate_feed.read(TEAMS * round_steps * a.gate.step);
        fetch(stage);
        stage = stage == my_ring ? my_ring + STAGE : my_ring;
        if (me.in_time) bar_sync<kTeam * 32>(kJoined + team);
        float2 h[P];
        get_state<TYPE>(h, here);
        if (valid > 0 && me.mine > 0) {
            if (a.starts) {
                float2* start = reinterpret_cast<float2*>(a.starts + (me.sequence * a.spans + t / kSpan) * a.starts_width + me.column + lane * LC);
#pragma unroll
                for (int p = 0; p < P; ++p) start[p] = h[p];
            }
            char* to = out;
            auto run = [&](auto whole) {
#pragma unroll
                for (int s = 0; s < kSpan; ++s) {
                    if (!whole.value && s >= valid) break;
#pragma unroll
                    for (int p = 0; p < P; ++p) h[p] = fma2(keep[s][p], h[p], zx[s][p]);
                    store_lane<TYPE, whole.value>(to, h, me.mine);
                    to += row;
                }
            };
            if (valid >= kSpan && a.whole) run(std::true_type()); else run(std::false_type());
        }
        out += TEAMS * round_steps * row;
        t += TEAMS * round_steps;
    }
    // The first warp that joined the last round has the state behind it.
    if (me.part == a.parts - 1 && me.in_time == 0 && team == (rounds ? (rounds - 1) % TEAMS : 0)) me.store_state(a.last, carry);
}

template <int TYPE, int UNIT, int TEAMS>
__global__ void __launch_bounds__(TEAMS * kTeam * 32, 2 / TEAMS) k_scan_back(ScanArgs a)
{
    extern __shared__ float4 room[];
    constexpr int P = kPairs<TYPE>, LC = kLaneChannels<TYPE>, STAGE = kStageBytes<UNIT, 3>;
    const int warp = (threadIdx.x >> 5) % kTeam, team = threadIdx.x / (kTeam * 32), lane = threadIdx.x & 31;
    char* ring = reinterpret_cast<char*>(room);
    float4* here = reinterpret_cast<float4*>(ring + TEAMS * kTeam * kStages * STAGE);
    float2* carried = reinterpret_cast<float2*>(here + TEAMS * P * kTeam * 32);
    here += team * P * kTeam * 32 + warp * 32 + lane;
    const Place<TYPE> me(a, warp);
    const uint32_t my_ring = shared_address(ring) + (threadIdx.x >> 5) * kStages * STAGE;
    const int begin = me.part * a.part_steps, end = min(a.steps, begin + a.part_steps), steps = me.live ? end : 0, round_steps = a.warps * kSpan;
    // Rounds go backward in time, as do the spans of each: from the segment's last one.
    int t = begin + ((end - begin + kSpan - 1) / kSpan - 1 - team * a.warps - me.in_time) * kSpan, fetched = t;      // first step of the span that comes next, and of the one fetched next
    Feed<TYPE, UNIT> x_feed(a.x, me.sequence, me.column, t, lane), gate_feed(a.gate, me.sequence, me.column, t, lane), dh_feed(a.dh, me.sequence, me.column, t, lane);
    auto valid_at = [&](int first) { return first < begin ? 0 : steps - first; };
    auto fetch = [&](uint32_t to) {
        const int valid = valid_at(fetched);
        x_feed.fetch(to, a.x, -TEAMS * round_steps * a.x.step, valid, me.channels, lane);
        gate_feed.fetch(to + kSpanBytes<UNIT>, a.gate, -TEAMS * round_steps * a.gate.step, valid, me.channels, lane);
        dh_feed.fetch(to + 2 * kSpanBytes<UNIT>, a.dh, -TEAMS * round_steps * a.dh.step, valid, me.channels, lane);
        fetched -= TEAMS * round_steps;
        copies_issued();
    };
    const float* starts = a.starts + (me.sequence * a.spans + t / kSpan) * a.starts_width + me.column + lane * LC;
    float2 start[P] = {};                                           // of the span that comes next
    auto fetch_start = [&](int first) {
        if (valid_at(first) > 0) {                                  // rows of starts hold whole slabs
#pragma unroll
            for (int p = 0; p < P; ++p) start[p] = reinterpret_cast<const float2*>(starts)[p];
        }
        starts -= TEAMS * a.warps * a.starts_width;
    };
#pragma unroll
    for (int r = 0; r < kStages; ++r) fetch(my_ring + r * STAGE);
    fetch_start(t);
    const int64_t row = a.width * kBytes<TYPE>, out = ((me.sequence * a.steps + t + kSpan - 1) * a.width + me.column + lane * LC) * kBytes<TYPE>;
    char *dx_out = static_cast<char*>(a.dx) + out, *dgate_out = static_cast<char*>(a.dgate) + out;       // of the span's last step
    uint32_t stage = my_ring;
    float2 carry[P];                                                // in the first warps in time
    me.load_state(carry, a.dlast);
#pragma unroll
    for (int p = 0; p < P; ++p) carry[p] = minus(carry[p]);         // with the other sign throughout: -G = -k - dh, dx = -z (-G), -k = -G + dx
    if (me.part < a.parts - 1 && me.in_time == 0 && team == 0) {
        wait_for_last_kernel();
        through_pieces<TYPE, Backward>(carry, me.piece(a, a.parts * a.pieces - 1), -P * 32, (a.parts - 1 - me.part) * a.pieces);
    }
    const int rounds = (end - begin + round_steps - 1) / round_steps;
    for (int round = team; round < rounds; round += TEAMS) {
        const int valid = valid_at(t);                              // 8 or more: the whole span
        const uint32_t from = stage + lane * 8;
        copies_done<kStages - 1>();
        __syncwarp();
        if (valid < kSpan) {                                        // behind the sequence nothing changes
#pragma unroll
            for (int s = 0; s < kSpan; ++s)
                if (s >= valid) { x_feed.zero(from, s, lane); dh_feed.zero(from + 2 * kSpanBytes<UNIT>, s, lane); }
            __syncwarp();
        }
        float2 nz[kSpan][P], az[kSpan][P];
#pragma unroll
        for (int s = 0; s < kSpan; ++s) {
            const uint2 g = gate_feed.words(from + kSpanBytes<UNIT>, s, a.gate);
#pragma unroll
            for (int p = 0; p < P; ++p) minus_taken_and_slope<TYPE>(pair_of<TYPE>(g, p), nz[s][p], az[s][p]);
        }
        if (valid < kSpan) {
#pragma unroll
            for (int s = 0; s < kSpan; ++s)
                if (s >= valid) {
#pragma unroll
                    for (int p = 0; p < P; ++p) nz[s][p] = az[s][p] = both(0.0f);
                }
        }
        Span mine[P];
#pragma unroll
        for (int p = 0; p < P; ++p) mine[p] = {both(0.0f), both(1.0f)};
#pragma unroll
        for (int s = kSpan - 1; s >= 0; --s) {
            const uint2 w = dh_feed.words(from + 2 * kSpanBytes<UNIT>, s, a.dh);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float2 g = sub2(mine[p].b, pair_of<TYPE>(w, p));
                mine[p].b = fma2(nz[s][p], g, g);
                mine[p].c = fma2(nz[s][p], mine[p].c, mine[p].c);
            }
        }
        put_span<TYPE>(mine, here);
        bar_sync<kTeam * 32>(kFormed + team);
        if (me.in_time == 0) {
            join_round<TYPE, Backward, TEAMS>(carry, round, rounds, a.warps, here, carried);
            bar_arrive<kTeam * 32>(kJoined + team);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) start[p] = minus(start[p]);
#pragma unroll
        for (int s = 0; s < kSpan; ++s) {                           // az becomes (x_t - h_(t-1)) a z; -h goes to (-h - z (-h)) - z x: of an h that z = 1 replaces nothing is left
            const uint2 w = x_feed.words(from, s, a.x);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float2 x = pair_of<TYPE>(w, p);
                az[s][p] = mul2(add2(x, start[p]), az[s][p]);
                start[p] = fma2(nz[s][p], x, fma2(nz[s][p], start[p], start[p]));
            }
        }
        fetch_start(t - TEAMS * round_steps);
        if (me.in_time) bar_sync<kTeam * 32>(kJoined + team);
        float2 k[P];
        get_state<TYPE>(k, here);
        if (valid > 0 && me.mine > 0) {
            char *dx = dx_out, *dgate = dgate_out;
            auto run = [&](auto whole) {
#pragma unroll
                for (int s = kSpan - 1; s >= 0; --s) {
                    const uint2 w = dh_feed.words(from + 2 * kSpanBytes<UNIT>, s, a.dh);
                    float2 v[P], u[P];
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const float2 g = sub2(k[p], pair_of<TYPE>(w, p));
                        v[p] = mul2(nz[s][p], g);
                        u[p] = mul2(g, az[s][p]);
                        k[p] = add2(g, v[p]);
                    }
                    if (whole.value || s < valid) {
                        store_lane<TYPE, whole.value>(dx, v, me.mine);
                        store_lane<TYPE, whole.value>(dgate, u, me.mine);
                    }
                    dx -= row;
                    dgate -= row;
                }
            };
            if (valid >= kSpan && a.whole) run(std::true_type()); else run(std::false_type());
        }
        __syncwarp();                                               // all lanes have read the stage
        x_feed.read(-TEAMS * round_steps * a.x.step);
        gate_feed.read(-TEAMS * round_steps * a.gate.step);
        dh_feed.read(-TEAMS * round_steps * a.dh.step);
        fetch(stage);
        stage = stage == my_ring ? my_ring + STAGE : my_ring;
        dx_out -= TEAMS * round_steps * row;
        dgate_out -= TEAMS * round_steps * row;
        t -= TEAMS * round_steps;
    }
    if (me.part == 0 && me.in_time == 0 && a.dstate && team == (rounds ? (rounds - 1) % TEAMS : 0)) {
#pragma unroll
        for (int p = 0; p < P; ++p) carry[p] = minus(carry[p]);
        me.store_state(a.dstate, carry);
    }
}

// What the segments but the last (backward: but the first) do to a state: a CTA takes a piece of a segment, each of its warps an eighth of that, joined at the end.
constexpr int kPartWarps = 8;
template <int TYPE, int UNIT, bool BACK>
__global__ void __launch_bounds__(kPartWarps * 32, 2) k_scan_parts(ScanArgs a)
{
    extern __shared__ float4 room[];
    using Way = std::conditional_t<BACK, Backward, Forward>;
    constexpr int P = kPairs<TYPE>, STAGE = kStageBytes<UNIT, 2>, STAGES = 3;
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = blockIdx.y + BACK * a.pieces;
    char* ring = reinterpret_cast<char*>(room);
    float4* here = reinterpret_cast<float4*>(ring + kPartWarps * STAGES * STAGE) + lane;
    const Place<TYPE> me(a, 0);
    const uint32_t my_ring = shared_address(ring) + warp * STAGES * STAGE;
    const int steps = a.part_steps / a.pieces, share = steps / kPartWarps, begin = piece * steps + warp * share, spans = share / kSpan;      // whole spans
    int fetched = begin + (BACK ? share - kSpan : 0);
    const Rows &one = BACK ? a.dh : a.x;
    Feed<TYPE, UNIT> feed(one, me.sequence, me.column, fetched, lane), gate_feed(a.gate, me.sequence, me.column, fetched, lane);
    int left = spans;
    auto fetch = [&](uint32_t to) {
        const int valid = left > 0 ? a.steps - fetched : 0;
        feed.fetch(to, one, (BACK ? -kSpan : kSpan) * one.step, valid, me.channels, lane);
        gate_feed.fetch(to + kSpanBytes<UNIT>, a.gate, (BACK ? -kSpan : kSpan) * a.gate.step, valid, me.channels, lane);
        fetched += BACK ? -kSpan : kSpan;
        --left;
        copies_issued();
    };
    int t = fetched;
#pragma unroll
    for (int r = 0; r < STAGES; ++r) fetch(my_ring + r * STAGE);
    uint32_t stage = my_ring;
    Span all[P];
    float2 all_product[P], all_forgotten[P];                        // forward
#pragma unroll
    for (int p = 0; p < P; ++p) {
        all[p] = {both(0.0f), both(1.0f)};
        all_product[p] = both(1.0f);
        all_forgotten[p] = both(0.0f);
    }
    for (int i = 0; i < spans; ++i) {
        const int valid = a.steps - t;
        const uint32_t from = stage + lane * 8;
        copies_done<STAGES - 1>();
        __syncwarp();
        Span mine[P];
        if constexpr (BACK) {
#pragma unroll
            for (int p = 0; p < P; ++p) mine[p] = {both(0.0f), both(1.0f)};
#pragma unroll
            for (int s = kSpan - 1; s >= 0; --s) {
                const uint2 w = feed.words(from, s, one), g = gate_feed.words(from + kSpanBytes<UNIT>, s, a.gate);
                if (s >= valid) continue;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float2 z = taken<TYPE>(pair_of<TYPE>(g, p)), nz = minus(z), sum = sub2(mine[p].b, pair_of<TYPE>(w, p));
                    mine[p].b = fma2(nz, sum, sum);
                    mine[p].c = fma2(nz, mine[p].c, mine[p].c);
                }
            }
#pragma unroll
            for (int p = 0; p < P; ++p) all[p] = Backward::join(all[p], mine[p]);
        } else {
            float2 keep[kSpan][P], zx[kSpan][P], product[P], forgotten[P];
            if (valid >= kSpan) form_span<TYPE, UNIT, true>(mine, product, forgotten, keep, zx, feed, gate_feed, a, from, valid);
            else form_span<TYPE, UNIT, false>(mine, product, forgotten, keep, zx, feed, gate_feed, a, from, valid);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                all[p].b = Forward::apply(mine[p], all[p].b);
                all_product[p] = mul2(product[p], all_product[p]);
                all_forgotten[p] = add2(forgotten[p], fma2(minus(forgotten[p]), all_forgotten[p], all_forgotten[p]));
            }
        }
        __syncwarp();                                               // all lanes have read the stage
        feed.read((BACK ? -kSpan : kSpan) * one.step);
        gate_feed.read((BACK ? -kSpan : kSpan) * a.gate.step);
        fetch(stage);
        stage = stage == my_ring + (STAGES - 1) * STAGE ? my_ring : stage + STAGE;
        t += BACK ? -kSpan : kSpan;
    }
    if constexpr (!BACK)
#pragma unroll
        for (int p = 0; p < P; ++p) all[p].c = Forward::choose(all_product[p], all_forgotten[p]);
#pragma unroll
    for (int p = 0; p < P; ++p) here[(warp * P + p) * 32] = make_float4(all[p].b.x, all[p].b.y, all[p].c.x, all[p].c.y);
    __syncthreads();
    if (warp == 0) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            Span s = span_of(here[((BACK ? kPartWarps - 1 : 0) * P + p) * 32]);
#pragma unroll
            for (int w = 1; w < kPartWarps; ++w) s = Way::join(s, span_of(here[((BACK ? kPartWarps - 1 - w : w) * P + p) * 32]));
            __stcg(me.piece(a, piece) + p * 32, make_float4(s.b.x, s.b.y, s.c.x, s.c.y));
        }
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

// Where z is above 1/2 as a span's steps are formed: 1 - z is exact, and the rounding of x - h, 2^-24 of a state that is gone, stays out of the new one.  Below, h + z (x - h) forgets nothing
// of a state to the rounding of 1 - z, however many tokens hold it.
__device__ __forceinline__ float step_of(float z, float x, float h) { return z > 0.5f ? fmaf(1.0f - z, h, z * x) : fmaf(z, x - h, h); }

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
    for (int j = 0; j < 8; ++j) h[j] = step_of(taken<TYPE>(make_float2(g[j], 0.0f)).x, x[j], h[j]);
    store8<APMS_GRAD_F32>(a.next, u * 8, h);
    store8<TYPE>(a.h, u * 8, h);
}

template <int TYPE>
__global__ void __launch_bounds__(128) k_scan_step_any(StepArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (i >= a.batch * a.width) return;
    const int64_t row = i / a.width, col = i - row * a.width;
    const float h = step_of(taken<TYPE>(make_float2(load1<TYPE>(a.gate, row * a.gate_stride + col), 0.0f)).x, load1<TYPE>(a.x, row * a.x_stride + col), a.state[i]);
    a.next[i] = h;
    store1<TYPE>(a.h, i, h);
}

// ------------------------------------------------------------------------------------------ host

// Warps in time: as many as the sequence has spans, up to a team.  Teams: two a CTA where the GPU's 148 SMs get no more than a slab each.  Segments: where they get fewer, as many as
// fill the SMs, one for every 128 steps at most, so that a sequence of 257 is cut already: 8 slabs of 511 bfloat16 steps take 10.5 us (backward 12.5), whole 12.5 (18.6); of 1024
// 10.6 (12.6), in segments of 512 at least 14.7 (20.4); of 257 9.0 (12.5) and 10.4 (12.9).  The one loss: the forward pass of 48 to 72 slabs of 257 to 384 steps, 12.5 us where a whole
// sequence takes 10.4.  By the sizes alone, so that results are the same on every GPU.
constexpr int kSms = 148, kLeastPart = 128;
int plan_scan(ScanArgs& a, int64_t batch, int64_t steps, int64_t width, int type)
{
    const int64_t wide = type == APMS_GRAD_F32 ? 64 : 128;
    a.batch = batch; a.steps = (int)steps; a.width = width;
    a.slabs = (width + wide - 1) / wide;
    a.spans = (a.steps + kSpan - 1) / kSpan;
    a.starts_width = (width + kStartsPad - 1) / kStartsPad * kStartsPad;
    a.warps = 1;
    while (a.warps < kTeam && a.warps < a.spans) a.warps *= 2;
    const int64_t sequences = std::max<int64_t>(1, batch * a.slabs), parts = std::max<int64_t>(1, std::min<int64_t>(kSms / sequences, steps / kLeastPart));
    a.parts = a.pieces = 1;
    a.part_steps = a.steps;
    if (parts > 1) {                                                // pieces: two CTAs an SM, or nearly so
        a.pieces = (int)std::min<int64_t>(4, 2 * kSms / (sequences * (parts - 1)));
        const int64_t unit = a.pieces == 3 ? 384 : a.pieces == 4 ? 256 : 128;                              // rounds of two teams, and spans for a piece's warps
        a.part_steps = (int)((steps + parts * unit - 1) / (parts * unit) * unit);
        a.parts = (int)((steps + a.part_steps - 1) / a.part_steps);
    }
    return sequences <= kSms && a.spans > kTeam ? 2 : 1;
}
size_t segment_bytes(const ScanArgs& a, int type) { return a.parts > 1 ? (size_t)(a.batch * a.slabs * a.parts * a.pieces) * (type == APMS_GRAD_F32 ? 1 : 2) * 32 * sizeof(float4) : 0; }

bool rows_on(const Rows& r, int64_t batch, int64_t steps, int64_t unit)
{
    return (uintptr_t)r.p % unit == 0 && (batch <= 1 || r.batch % unit == 0) && (steps <= 1 || r.step % unit == 0);
}

template <int TYPE, int UNIT, bool BACK>
cudaError_t launch_scan_unit(const ScanArgs& a, int teams, cudaStream_t stream)
{
    auto one = BACK ? k_scan_back<TYPE, UNIT, 1> : k_scan<TYPE, UNIT, 1>, two = BACK ? k_scan_back<TYPE, UNIT, 2> : k_scan<TYPE, UNIT, 2>;
    auto parts = k_scan_parts<TYPE, UNIT, BACK>;
    constexpr int TENSORS = BACK ? 3 : 2, P = kPairs<TYPE>;
    constexpr size_t part_shared = (size_t)kPartWarps * (3 * kStageBytes<UNIT, 2> + P * 32 * sizeof(float4));
    static Raised raised[3][kMostDevices];
    cudaError_t e = raise_limits(raised[0], reinterpret_cast<const void*>(one), scan_shared<UNIT, TENSORS>(1, P), false);
    if (e == cudaSuccess) e = raise_limits(raised[1], reinterpret_cast<const void*>(two), scan_shared<UNIT, TENSORS>(2, P), false);
    if (e == cudaSuccess) e = raise_limits(raised[2], reinterpret_cast<const void*>(parts), part_shared, false);
    if (e != cudaSuccess) return e;
    if (a.parts > 1) {
        e = launch(parts, dim3((unsigned)(a.batch * a.slabs), (unsigned)((a.parts - 1) * a.pieces)), kPartWarps * 32, part_shared, stream, false, a);
        if (e != cudaSuccess) return e;
    }
    const int64_t per_cta = kTeam / a.warps;
    const dim3 grid((unsigned)((a.batch * a.slabs + per_cta - 1) / per_cta), (unsigned)a.parts);
    return launch(teams == 2 ? two : one, grid, teams * kTeam * 32, scan_shared<UNIT, TENSORS>(teams, P), stream, a.parts > 1, a);
}

template <int TYPE, bool BACK>
cudaError_t launch_scan(const ScanArgs& a, int teams, cudaStream_t stream)
{
    constexpr int64_t ES = kBytes<TYPE>;
    auto on = [&](int64_t unit) {
        return a.width * ES % unit == 0 && rows_on(a.x, a.batch, a.steps, unit) && rows_on(a.gate, a.batch, a.steps, unit) && (!BACK || rows_on(a.dh, a.batch, a.steps, unit));
    };
    if (on(16)) return launch_scan_unit<TYPE, 16, BACK>(a, teams, stream);
    if (ES == 4 || on(4)) return launch_scan_unit<TYPE, 4, BACK>(a, teams, stream);
    if constexpr (ES == 2) return launch_scan_unit<TYPE, 2, BACK>(a, teams, stream);
    return cudaErrorInvalidValue;
}

template <bool BACK>
cudaError_t launch_scan_types(const ScanArgs& a, int type, int teams, cudaStream_t stream)
{
    return type == APMS_GRAD_F32 ? launch_scan<APMS_GRAD_F32, BACK>(a, teams, stream)
         : type == APMS_GRAD_BF16 ? launch_scan<APMS_GRAD_BF16, BACK>(a, teams, stream) : launch_scan<APMS_GRAD_F16, BACK>(a, teams, stream);
}

template <int TYPE>
cudaError_t launch_step(const StepArgs& a, bool vector, cudaStream_t stream)
{
    const int64_t n = vector ? a.batch * a.width / 8 : a.batch * a.width;
    return launch(vector ? k_scan_step<TYPE> : k_scan_step_any<TYPE>, dim3((unsigned)((n + 127) / 128)), 128, 0, stream, false, a);
}

constexpr int64_t kMostScan = (int64_t)1 << 31, kMostSteps = (int64_t)1 << 30, kMostScanElements = (int64_t)1 << 40;

bool scan_sizes(int64_t batch, int64_t steps, int64_t width)
{
    return batch >= 0 && steps >= 0 && width >= 1 && batch < kMostScan && steps <= kMostSteps && width < kMostScan && batch * width <= kMostScan && batch * width * steps <= kMostScanElements;
}

apms_status scan_check(const char* who, int64_t batch, int64_t steps, int64_t width, apms_grad_type type)
{
    if (!scan_sizes(batch, steps, width))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld sequences of %lld steps of %lld channels: needs none below 0, width >= 1, steps <= 2^30, batch * width <= 2^31 and at most 2^40 elements", who,
                             (long long)batch, (long long)steps, (long long)width);
    if (!known_type(type)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: unknown element type", who);
    return APMS_OK;
}

}  // namespace

extern "C" {

size_t apms_gated_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t width, apms_grad_type type)
{
    if (!scan_sizes(batch, steps, width) || !known_type(type)) return 0;
    ScanArgs a = {};
    plan_scan(a, batch, steps, width, type);
    return segment_bytes(a, type);
}

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
    if (!on_element(g.x, g.type) || !on_element(g.gate, g.type) || !on_element(g.h, g.type) || !on_element(g.state, APMS_GRAD_F32) || !on_element(g.last, APMS_GRAD_F32) || !on_16(g.starts))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    ScanArgs a = {};
    const int64_t es = (int64_t)element_size(g.type);
    const int teams = plan_scan(a, g.batch, g.steps, g.width, g.type);
    if (a.parts > 1 && (!g.workspace_dev || !on_16(g.workspace_dev) || g.workspace_bytes < segment_bytes(a, g.type)))
        return operator_fail(APMS_ERR_OOM, "%s: needs apms_gated_scan_workspace_bytes() of 16-byte aligned workspace", who);
    a.segments = static_cast<float4*>(g.workspace_dev);
    a.x = {g.x, g.x_batch_stride * es, g.x_step_stride * es};
    a.gate = {g.gate, g.gate_batch_stride * es, g.gate_step_stride * es};
    a.state = g.state; a.h = g.h; a.last = g.last; a.starts = g.starts;
    a.whole = a.width * es % 8 == 0 && (uintptr_t)a.h % 8 == 0;
    const cudaError_t e = launch_scan_types<false>(a, g.type, teams, (cudaStream_t)cuda_stream);
    OPERATOR_CUDA("apms_gated_scan", e);
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
        !on_16(g.starts) || !on_element(g.dlast, APMS_GRAD_F32) || !on_element(g.dstate, APMS_GRAD_F32))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    ScanArgs a = {};
    const int64_t es = (int64_t)element_size(g.type);
    const int teams = plan_scan(a, g.batch, g.steps, g.width, g.type);
    if (a.parts > 1 && (!g.workspace_dev || !on_16(g.workspace_dev) || g.workspace_bytes < segment_bytes(a, g.type)))
        return operator_fail(APMS_ERR_OOM, "%s: needs apms_gated_scan_workspace_bytes() of 16-byte aligned workspace", who);
    a.segments = static_cast<float4*>(g.workspace_dev);
    a.x = {g.x, g.x_batch_stride * es, g.x_step_stride * es};
    a.gate = {g.gate, g.gate_batch_stride * es, g.gate_step_stride * es};
    a.dh = {g.dh, g.dh_batch_stride * es, g.dh_step_stride * es};
    a.starts = const_cast<float*>(g.starts); a.dlast = g.dlast; a.dx = g.dx; a.dgate = g.dgate; a.dstate = g.dstate;
    a.whole = a.width * es % 8 == 0 && (uintptr_t)a.dx % 8 == 0 && (uintptr_t)a.dgate % 8 == 0;
    const cudaError_t e = launch_scan_types<true>(a, g.type, teams, (cudaStream_t)cuda_stream);
    OPERATOR_CUDA("apms_gated_scan_backward", e);
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
    const bool vector = rows_of_eight(a.x, a.batch, a.x_stride, a.width, g.type) && rows_of_eight(a.gate, a.batch, a.gate_stride, a.width, g.type) && on_eight(a.h, g.type) && on_eight(a.state, APMS_GRAD_F32) && on_eight(a.next, APMS_GRAD_F32);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    OPERATOR_CUDA("apms_gated_scan_step", g.type == APMS_GRAD_F32 ? launch_step<APMS_GRAD_F32>(a, vector, stream)
                                        : g.type == APMS_GRAD_BF16 ? launch_step<APMS_GRAD_BF16>(a, vector, stream) : launch_step<APMS_GRAD_F16>(a, vector, stream));
    return APMS_OK;
}

}  // extern "C"
