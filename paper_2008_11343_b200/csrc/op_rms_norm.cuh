// Root-mean-square norm at a residual junction, with 8-bit output, and its gradient.
// Part of libapms.so: included by operators.cu.
//
//   h = x + r,  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd w                      (per row)
//   xh = h rstd,  a = w dy,  dx = rstd (a - xh mean(a xh)) + dh,  dw = sum_rows dy xh
//
// All streams: 6 operations per element forwards, 12 backwards.  In 16 bits the instructions (18 to 26 an element, most of them widening and
// packing) keep the issue slots half busy beside HBM, so these kernels follow the SM clock too: figures are at the 1.7 to 1.9 GHz
// of a long run unless they say otherwise.
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
    float eps, inv_width;
};

// |v| as bits: ordered like the magnitudes, with infinity and then NaN above every number, so a maximum keeps NaN
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ float max_nan(float a, float b)          // NaN where either is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float warp_most(float v, int lanes)       // over groups of `lanes` lanes
{
    for (int o = lanes / 2; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A group's scale and what its elements are multiplied by.
__device__ __forceinline__ void group_scale(uint32_t most_bits, float* scale, float* inverse)
{
    const float a = __uint_as_float(most_bits);
    const bool none = a < kScaleFloor;
    *scale = none ? 0.0f : __fdiv_rn(a, kE4m3Max);
    *inverse = none ? 0.0f : __fdiv_rn(kE4m3Max, a);
}

// How a warp lays its elements of a row over its lanes.  VECTOR: 16 bytes of the activations' type a lane (8 or 4 consecutive
// elements), for rows that all start on a 16-byte boundary and hold whole 16-byte pieces.  Otherwise 4 elements a lane, 32 apart, so
// that the accesses of a warp are consecutive.  A unit is what a warp's lanes hold at one time: 128 or 256 elements; a
// group of 128 columns is then always a whole warp or half of one.
template <int XT, bool VECTOR>
struct Lanes {
    static constexpr int E = VECTOR && XT != APMS_GRAD_F32 ? 8 : 4;      // elements a lane and unit
    static constexpr int UNIT = 32 * E, GROUP_LANES = 128 / E;
    // column of element j of a lane in a unit of the row
    static __device__ __forceinline__ int column(int unit, int lane, int j) { return unit * UNIT + (VECTOR ? lane * E + j : lane + 32 * j); }
};

// Elements from the words they lie in, in pairs.
template <int TYPE, int WORDS>
__device__ __forceinline__ void unpack_words(float2* f, const uint32_t* w)
{
    if (TYPE == APMS_GRAD_F32) {
#pragma unroll
        for (int k = 0; k < WORDS; k += 2) f[k / 2] = make_float2(__uint_as_float(w[k]), __uint_as_float(w[k + 1]));
    } else {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) f[k] = unpack16<TYPE == APMS_GRAD_F32 ? APMS_GRAD_BF16 : TYPE>(w[k]);
    }
}

// E elements of type TYPE of a unit of the row, in pairs; 0 behind the width.
template <int TYPE, class L, bool VECTOR>
__device__ __forceinline__ void load_unit(float2* f, const char* row, int unit, int lane, int width)
{
    constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2, WORDS = L::E * ES / 4;
    if (VECTOR) {
        const int c = L::column(unit, lane, 0);
        uint32_t w[WORDS];
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] = 0;
        if (c < width) {
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) load16(w + k, row + c * ES + 4 * k);
        }
        unpack_words<TYPE, WORDS>(f, w);
    } else {
#pragma unroll
        for (int j = 0; j < L::E; j += 2) {
            const int c = L::column(unit, lane, j), c1 = L::column(unit, lane, j + 1);
            f[j / 2].x = c < width ? load_element(row, c, TYPE) : 0.0f;
            f[j / 2].y = c1 < width ? load_element(row, c1, TYPE) : 0.0f;
        }
    }
}

// H pairs as TYPE (rounded once) or as e4m3, at an address aligned to their bytes (16 at most).
template <int TYPE, int H>
__device__ __forceinline__ void store_pairs(char* p, const float2* f)
{
    if (TYPE == APMS_GRAD_F32) {
#pragma unroll
        for (int k = 0; k < H; k += 2) *reinterpret_cast<float4*>(p + 8 * k) = make_float4(f[k].x, f[k].y, f[k + 1].x, f[k + 1].y);
    } else {
        constexpr int T = TYPE == APMS_GRAD_F32 ? APMS_GRAD_BF16 : TYPE;
        if (H == 4) *reinterpret_cast<uint4*>(p) = make_uint4(pack16<T>(f[0]), pack16<T>(f[1]), pack16<T>(f[2 % H]), pack16<T>(f[3 % H]));
        else *reinterpret_cast<uint2*>(p) = make_uint2(pack16<T>(f[0]), pack16<T>(f[1]));
    }
}
template <int H>
__device__ __forceinline__ void store_e4m3(char* p, const float2* f)
{
    uint32_t w[H / 2];
#pragma unroll
    for (int k = 0; k < H / 2; ++k)
        w[k] = (uint32_t)__nv_cvt_float2_to_fp8x2(f[2 * k], __NV_SATFINITE, __NV_E4M3) | (uint32_t)__nv_cvt_float2_to_fp8x2(f[2 * k + 1], __NV_SATFINITE, __NV_E4M3) << 16;
    if (H == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[H / 2 - 1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
}

template <int TYPE, class L, bool VECTOR>
__device__ __forceinline__ void store_unit(char* row, const float2* f, int unit, int lane, int width)
{
    constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2;
    if (VECTOR) {
        const int c = L::column(unit, lane, 0);
        if (c < width) store_pairs<TYPE, L::E / 2>(row + c * ES, f);
    } else {
#pragma unroll
        for (int j = 0; j < L::E; ++j) {
            const int c = L::column(unit, lane, j);
            if (c < width) store_element(row, c, TYPE, j & 1 ? f[j / 2].y : f[j / 2].x);
        }
    }
}

constexpr int kTeamWarps = 16;                   // a row's at most

// 16 bytes from global to shared memory without a register; both 16-byte aligned.  A thread copies what it reads itself,
// so its own wait is all the order that is needed.
__device__ __forceinline__ void copy16_async(uint32_t to_shared, const char* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to_shared), "l"(from) : "memory");
}
__device__ __forceinline__ void put_zeros(uint32_t shared) { asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" :: "r"(shared), "r"(0) : "memory"); }
__device__ __forceinline__ void load_shared16(uint32_t* w, uint32_t shared)
{
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(shared) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_for_copies() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

// copies `bytes` (1 to 16) of the 16, the rest become zeros
__device__ __forceinline__ void copy16_async(char* to_shared, const char* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"((uint32_t)__cvta_generic_to_shared(to_shared)), "l"(from), "r"(bytes) : "memory");
}

// A row of `count` elements of ES bytes at p into `room`, by the `threads` threads of a team; where its first element will be.
template <int ES>
__device__ __forceinline__ const char* stage_shifted(char* room, const char* p, int count, int t, int threads)
{
    const int shift = (int)((uintptr_t)p & 15);
    const char* from = p - shift;
    const int bytes = shift + count * ES;            // of the pieces from `from` on
    const int first = shift ? 1 : 0;
    if (first && t < (16 - shift) / ES && t < count) {
        if (ES == 4) reinterpret_cast<uint32_t*>(room + shift)[t] = reinterpret_cast<const uint32_t*>(p)[t];
        else reinterpret_cast<uint16_t*>(room + shift)[t] = reinterpret_cast<const uint16_t*>(p)[t];
    }
    for (int k = first + t; k * 16 < bytes; k += threads) copy16_async(room + k * 16, from + k * 16, min(16, bytes - k * 16));
    return room + shift;
}

// What the warps of a row (blockDim.x threads, a row per threadIdx.y) found in its first reading, over the row, in every thread: the sum of squares, and the
// largest magnitude where it is wanted.  Every thread of the CTA calls it.  smem: 2 kTeamWarps floats.
__device__ __forceinline__ void join_team(float& squares, float& most, bool take_most, float* smem)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team_warps = blockDim.x >> 5;
    squares = warp_total(squares);
    if (take_most) most = warp_most(most, 32);
    if (team_warps == 1) return;
    float* team = smem + threadIdx.y * team_warps;
    if (lane == 0) { team[warp] = squares; team[kTeamWarps + warp] = most; }
    __syncthreads();
    squares = team[0];
    for (int w = 1; w < team_warps; ++w) squares += team[w];
    if (take_most) {
        most = team[kTeamWarps];
        for (int w = 1; w < team_warps; ++w) most = max_nan(most, team[kTeamWarps + w]);
    }
}

// One element in shared memory.
template <int TYPE>
__device__ __forceinline__ float load_shared_element(uint32_t shared)
{
    if (TYPE == APMS_GRAD_F32) {
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(shared) : "memory");
        return v;
    }
    unsigned short v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(shared) : "memory");
    return unpack16<TYPE == APMS_GRAD_F32 ? APMS_GRAD_BF16 : TYPE>(v).x;
}
template <int ES>
__device__ __forceinline__ void put_zero_element(uint32_t shared)
{
    if (ES == 4) asm volatile("st.shared.u32 [%0], %1;" :: "r"(shared), "r"(0) : "memory");
    else asm volatile("st.shared.u16 [%0], %1;" :: "r"(shared), "h"((unsigned short)0) : "memory");
}

// Narrow rows (up to 256 elements of 16 bits, 128 of 32), whole 16-byte pieces: TL lanes a row and R rows a lane, in registers, the weight loaded once for
// them: 200,000 x 128 bfloat16 35 us = 5.9 TB/s.  A row a warp left half its lanes without work there and 32 bytes a lane in flight: 68 us.
template <int XT, int RT, int WT, int TL>
__global__ void __launch_bounds__(128)
k_rms_narrow(const RmsArgs a, int64_t rows)
{
    using L = Lanes<XT, true>;
    constexpr int E = L::E, H = E / 2, R = 4, XS = XT == APMS_GRAD_F32 ? 4 : 2, RS = RT == APMS_GRAD_F32 ? 4 : 2;
    constexpr int GROUP = L::GROUP_LANES < TL ? L::GROUP_LANES : TL;
    const int lane = threadIdx.x % TL, c = lane * E, width = (int)a.width;
    const int64_t row0 = ((int64_t)blockIdx.x * (128 / TL) + threadIdx.x / TL) * R;
    float2 h[R][H], w[H];
#pragma unroll
    for (int k = 0; k < R; ++k) load_unit<XT, L, true>(h[k], static_cast<const char*>(a.x) + (row0 + k) * a.x_stride * XS, 0, lane, row0 + k < rows ? width : 0);
    if (a.r) {
        float2 r[R][H];
#pragma unroll
        for (int k = 0; k < R; ++k) load_unit<RT, L, true>(r[k], static_cast<const char*>(a.r) + (row0 + k) * a.r_stride * RS, 0, lane, row0 + k < rows ? width : 0);
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int j = 0; j < H; ++j) h[k][j] = add2(h[k][j], r[k][j]);
    }
    load_unit<WT, L, true>(w, static_cast<const char*>(a.w), 0, lane, width);
    const bool row_scale = a.scales && a.group == a.width;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int64_t row = row0 + k;
        const int in = row < rows ? width : 0;
        float2 acc = both(0.0f);
#pragma unroll
        for (int j = 0; j < H; ++j) acc = fma2(h[k][j], h[k][j], acc);
        float squares = acc.x + acc.y;
#pragma unroll
        for (int o = TL / 2; o > 0; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
        const float rstd = rsqrtf(squares * a.inv_width + a.eps);
        if (lane == 0 && in) a.rstd[row] = rstd;
        if (a.r) store_unit<RT, L, true>(static_cast<char*>(a.h) + row * a.width * RS, h[k], 0, lane, in);
#pragma unroll
        for (int j = 0; j < H; ++j) h[k][j] = mul2(mul2(h[k][j], both(rstd)), w[j]);
        if (!a.scales) {
            store_unit<XT, L, true>(static_cast<char*>(a.y) + row * a.width * XS, h[k], 0, lane, in);
            continue;
        }
        float m = 0.0f, scale, inverse;
#pragma unroll
        for (int j = 0; j < H; ++j) m = max_nan(m, max_nan(fabsf(h[k][j].x), fabsf(h[k][j].y)));
        m = warp_most(c < in ? m : 0.0f, row_scale ? TL : GROUP);
        group_scale(magnitude_bits(m), &scale, &inverse);
        if (c < in && lane % (row_scale ? TL : GROUP) == 0) a.scales[row * a.groups + (row_scale ? 0 : c / 128)] = scale;
#pragma unroll
        for (int j = 0; j < H; ++j) h[k][j] = mul2(h[k][j], both(inverse));
        if (c < in) store_e4m3<H>(static_cast<char*>(a.y) + row * a.width + c, h[k]);
    }
}

// Rows of whole 16-byte pieces, through shared memory: x and the residual are copied there without registers, each thread copying what it
// reads itself, and read twice - for the sums, and for the outputs.  Little of the row stays in registers, so more of it is in flight on an
// SM: with the row in registers (binary32 beside the weight) 16384x4096 bfloat16 to 8 bits took 100 us in short runs, so 72 us; a CTA ends
// with its row or rows, the next CTAs' copies cover the latency of its sum (persistent CTAs with a ring of rows: 87 us).  8192x4096
// bfloat16 with a residual: 44.2 us = 6.1 TB/s, binary32 83.6 us = 6.4 TB/s, to 8 bits (16384 rows) 76.0 us = 6.2 TB/s.
// The row's 8-bit scale comes from max |h weight|, which the first reading can take: |y| is that times rstd, up to one rounding.
// RES: with a residual.  Two rows a team, to share the indexes and the weight, were slower (45.1 against 47.0 us): fewer CTAs.
template <int XT, int RT, int WT, bool RES, int NU>
__global__ void __launch_bounds__(kTeamWarps * 32)
k_rms_staged(const RmsArgs a, int64_t rows)
{
    using L = Lanes<XT, true>;
    constexpr int E = L::E, H = E / 2, XS = XT == APMS_GRAD_F32 ? 4 : 2, RS = RT == APMS_GRAD_F32 ? 4 : 2, WS = WT == APMS_GRAD_F32 ? 4 : 2;
    constexpr int DR = RES ? E * RS / 16 : 0, WORDS = E * WS / 4;
    extern __shared__ __align__(16) char staged[];
    __shared__ float red[2 * kTeamWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = warp * (NU * L::UNIT) + lane * E, width = (int)a.width;        // unit u of this lane begins at c0 + u UNIT
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int in = row < rows ? width : 0;           // a team without a row loads nothing and stays for the barrier
    const int piece = 16 * blockDim.x * blockDim.y, per_unit = piece * (1 + DR);
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(staged) + 16 * (threadIdx.y * blockDim.x + threadIdx.x);      // a unit's pieces: x, then the residual's
    const char* xp = static_cast<const char*>(a.x) + row * a.x_stride * XS + c0 * XS;
    const char* rp = static_cast<const char*>(a.r) + row * a.r_stride * RS + c0 * RS;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const uint32_t to = mine + u * per_unit;
        if (c0 + u * L::UNIT < in) {
            copy16_async(to, xp + u * (L::UNIT * XS));
#pragma unroll
            for (int j = 0; j < DR; ++j) copy16_async(to + (1 + j) * piece, rp + u * (L::UNIT * RS) + 16 * j);
        } else {                                     // zeros, so that the sums need not ask
#pragma unroll
            for (int j = 0; j < 1 + DR; ++j) put_zeros(to + j * piece);
        }
    }
    commit_copies();
    uint32_t weight[NU][WORDS];
    auto load_weight = [&]() {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
#pragma unroll
            for (int k = 0; k < WORDS; ++k) weight[u][k] = 0;
            if (c0 + u * L::UNIT < in) {
#pragma unroll
                for (int k = 0; k < WORDS; k += 4) load16(weight[u] + k, static_cast<const char*>(a.w) + c0 * WS + u * (L::UNIT * WS) + 4 * k);
            }
        }
    };
    auto h_of = [&](float2* h, int u) {
        const uint32_t from = mine + u * per_unit;
        uint32_t w[8];
        load_shared16(w, from);
        unpack_words<XT, E * XS / 4>(h, w);
        if (RES) {
            float2 r[H];
#pragma unroll
            for (int j = 0; j < DR; ++j) load_shared16(w + 4 * j, from + (1 + j) * piece);
            unpack_words<RT, E * RS / 4>(r, w);
#pragma unroll
            for (int j = 0; j < H; ++j) h[j] = add2(h[j], r[j]);
        }
    };
    const bool row_scale = a.scales && a.group == a.width;
    float2 acc = both(0.0f);
    float most = 0.0f;
    if (row_scale) {
        load_weight();
        wait_for_copies<0>();
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float2 h[H], w[H];
            h_of(h, u);
            unpack_words<WT, WORDS>(w, weight[u]);
#pragma unroll
            for (int j = 0; j < H; ++j) {
                acc = fma2(h[j], h[j], acc);
                const float2 v = mul2(h[j], w[j]);
                most = max_nan(most, max_nan(fabsf(v.x), fabsf(v.y)));
            }
        }
    } else {
        wait_for_copies<0>();
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float2 h[H];
            h_of(h, u);
#pragma unroll
            for (int j = 0; j < H; ++j) acc = fma2(h[j], h[j], acc);
        }
        load_weight();                               // while the sums are under way
    }
    float squares = acc.x + acc.y;
    join_team(squares, most, row_scale, red);
    const float rstd = rsqrtf(squares * a.inv_width + a.eps);
    float scale = 0.0f, inverse = 0.0f;
    if (row_scale) group_scale(magnitude_bits(most * rstd), &scale, &inverse);
    if (threadIdx.x == 0 && in) {
        a.rstd[row] = rstd;
        if (row_scale) a.scales[row] = scale;
    }
    char* hr = static_cast<char*>(a.h) + (row * width + c0) * RS;
    char* yr = static_cast<char*>(a.y) + (row * width + c0) * (a.scales ? 1 : XS);
    if (!a.scales) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float2 h[H], w[H];
            unpack_words<WT, WORDS>(w, weight[u]);
            h_of(h, u);
            const bool inside = c0 + u * L::UNIT < in;
            if (RES && inside) store_pairs<RT, H>(hr + u * (L::UNIT * RS), h);
#pragma unroll
            for (int j = 0; j < H; ++j) h[j] = mul2(mul2(h[j], both(rstd)), w[j]);
            if (inside) store_pairs<XT, H>(yr + u * (L::UNIT * XS), h);
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const bool inside = c0 + u * L::UNIT < in;
        float2 h[H], w[H];
        unpack_words<WT, WORDS>(w, weight[u]);
        h_of(h, u);
        if (RES && inside) store_pairs<RT, H>(hr + u * (L::UNIT * RS), h);
#pragma unroll
        for (int j = 0; j < H; ++j) h[j] = mul2(mul2(h[j], both(rstd)), w[j]);
        if (!row_scale) {                            // 128 columns: a warp or half of one
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < H; ++j) m = max_nan(m, max_nan(fabsf(h[j].x), fabsf(h[j].y)));
            m = warp_most(inside ? m : 0.0f, L::GROUP_LANES);                     // zeros are NaN by now where rstd is infinite or NaN
            group_scale(magnitude_bits(m), &scale, &inverse);
            if (lane % L::GROUP_LANES == 0 && inside) a.scales[row * a.groups + (c0 + u * L::UNIT) / 128] = scale;
        }
#pragma unroll
        for (int j = 0; j < H; ++j) h[j] = mul2(h[j], both(inverse));
        if (inside) store_e4m3<H>(yr + u * L::UNIT, h);
    }
}

// Rows that do not start on 16-byte boundaries or hold a ragged number of bytes, through shared memory too: the 16-byte pieces that a row touches are
// copied as they lie (its first bytes, up to a boundary, by plain loads: what is before them may not be the caller's), and
// its elements read one by one from there, 32 lanes' consecutive.  Bound by those 2-byte accesses: 8192 x 1001 bfloat16 24 us = 2.7 TB/s
// (2-byte loads from global memory: 28 us), 4000 x 8191 82 us = 3.2 TB/s.
template <int XT, int RT, int WT, bool RES, int NU>
__global__ void __launch_bounds__(kTeamWarps * 32)
k_rms_shifted(const RmsArgs a, int64_t rows, int x_room, int r_room)
{
    using L = Lanes<XT, false>;
    constexpr int E = L::E, XS = XT == APMS_GRAD_F32 ? 4 : 2, RS = RT == APMS_GRAD_F32 ? 4 : 2, WS = WT == APMS_GRAD_F32 ? 4 : 2;
    extern __shared__ __align__(16) char staged[];
    __shared__ float red[2 * kTeamWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team_warps = blockDim.x >> 5, width = (int)a.width;
    const int c0 = warp * (NU * L::UNIT) + lane, padded = team_warps * (NU * L::UNIT);        // element j of unit u of this lane: column c0 + 128 u + 32 j
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int in = row < rows ? width : 0, left = in - c0;
    char* room = staged + threadIdx.y * (x_room + r_room);
    const char* xs = stage_shifted<XS>(room, static_cast<const char*>(a.x) + row * a.x_stride * XS, in, threadIdx.x, blockDim.x);
    const char* rs = RES ? stage_shifted<RS>(room + x_room, static_cast<const char*>(a.r) + row * a.r_stride * RS, in, threadIdx.x, blockDim.x) : xs;
    commit_copies();
    float w[NU][E];
    const char* wp = static_cast<const char*>(a.w) + (int64_t)c0 * WS;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < E; ++j) w[u][j] = u * L::UNIT + 32 * j < left ? load_element(wp + (u * L::UNIT + 32 * j) * WS, 0, WT) : 0.0f;
    const bool row_scale = a.scales && a.group == a.width;
    wait_for_copies<0>();
    for (int c = in + threadIdx.x; c < padded; c += blockDim.x) {       // zeros behind the row, so that the sums need not ask
        put_zero_element<XS>((uint32_t)__cvta_generic_to_shared(xs) + c * XS);
        if (RES) put_zero_element<RS>((uint32_t)__cvta_generic_to_shared(rs) + c * RS);
    }
    __syncthreads();
    const uint32_t xa = (uint32_t)__cvta_generic_to_shared(xs) + c0 * XS, ra = (uint32_t)__cvta_generic_to_shared(rs) + c0 * RS;
    auto h_of = [&](int k) {                         // of column c0 + k
        const float h = load_shared_element<XT>(xa + k * XS);
        return RES ? h + load_shared_element<RT>(ra + k * RS) : h;
    };
    float squares = 0.0f, most = 0.0f;
    if (row_scale) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float h = h_of(u * L::UNIT + 32 * j);
                squares = fmaf(h, h, squares);
                most = max_nan(most, fabsf(h * w[u][j]));
            }
    } else {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float h = h_of(u * L::UNIT + 32 * j);
                squares = fmaf(h, h, squares);
            }
    }
    join_team(squares, most, row_scale, red);
    const float rstd = rsqrtf(squares * a.inv_width + a.eps);
    float scale = 0.0f, inverse = 0.0f;
    if (row_scale) group_scale(magnitude_bits(most * rstd), &scale, &inverse);
    if (threadIdx.x == 0 && in) {
        a.rstd[row] = rstd;
        if (row_scale) a.scales[row] = scale;
    }
    char* hp = static_cast<char*>(a.h) + (row * width + c0) * RS;
    char* yp = static_cast<char*>(a.y) + (row * width + c0) * (a.scales ? 1 : XS);
    if (!a.scales) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int k = u * L::UNIT + 32 * j;
                const float h = h_of(k);
                if (k < left) {
                    if (RES) store_element(hp + k * RS, 0, RT, h);
                    store_element(yp + k * XS, 0, XT, h * rstd * w[u][j]);
                }
            }
        return;
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        float y[E], m = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int k = u * L::UNIT + 32 * j;
            const float h = h_of(k);
            y[j] = h * rstd * w[u][j];
            if (k < left) {
                if (RES) store_element(hp + k * RS, 0, RT, h);
                m = max_nan(m, fabsf(y[j]));         // zeros behind the row are NaN by now where rstd is infinite or NaN
            }
        }
        if (!row_scale) {
            group_scale(magnitude_bits(warp_most(m, 32)), &scale, &inverse);
            if (lane == 0 && u * L::UNIT < left) a.scales[row * a.groups + (c0 + u * L::UNIT) / 128] = scale;
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int k = u * L::UNIT + 32 * j;
            if (k < left) yp[k] = (char)__nv_cvt_float_to_fp8(y[j] * inverse, __NV_SATFINITE, __NV_E4M3);
        }
    }
}

// Rows that do not fit into a team's units or a CTA's shared memory (wider than 65,536 in 16 bits, 53,248 with a residual, 36,864 with a binary32 one, 32,768
// in binary32, 26,624 with a residual; off the 16-byte boundary 32,768, and 26,624 in binary32 with a residual): one CTA per row, any stride and alignment, read again for each pass.  A thread adds
// width / 256 squares one after the other, up to 65,536: in binary64 (1 % of the time; binary32: rstd off by up to 356 units in the last place on
// equal elements, 2^20 wide).
__global__ void __launch_bounds__(kRmsThreads)
k_rms_rows(const RmsArgs a)
{
    __shared__ double red[kRmsThreads / 32];
    __shared__ uint32_t most;
    const int64_t row = blockIdx.x;
    const int64_t x0 = row * a.x_stride, r0 = row * a.r_stride, o0 = row * a.width;
    auto h_of = [&](int64_t c) {
        float h = load_element(a.x, x0 + c, a.x_type);
        return a.r ? h + load_element(a.r, r0 + c, a.r_type) : h;
    };
    double acc = 0.0;
    for (int64_t c = threadIdx.x; c < a.width; c += kRmsThreads) {
        const double h = (double)h_of(c);
        acc = fma(h, h, acc);
    }
    const float rstd = rsqrtf((float)block_total(acc, red) * a.inv_width + a.eps);
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
    float inv_width;
};

// A CTA walks over rows, a team of warps each, and keeps its columns' share of dweight in registers; `partial` gets one row of shares per CTA.
// The rows' operands come through a ring of STAGES rows in shared memory, copied ahead (cp.async: neither registers nor a
// producer), because one row a CTA in flight at a time would not cover HBM's latency.
// VECTOR: rows of whole 16-byte pieces; each thread copies what it reads itself, so a row costs one barrier, its sum's.
// Otherwise the pieces a row touches are copied as they lie, by the team together, and read one element at a time: a barrier more a row.
// 16384x4096 bfloat16 with dh 87.8 us = 6.1 TB/s (19 instructions an element), 8192x1001 27 us; with a binary32 stream, 160 bytes a thread and
// stage leave two stages: 8192x4096 123 us = 4.3 TB/s.
template <int XT, int HT, bool VECTOR, int NU>
struct BackShape {
    using L = Lanes<XT, VECTOR>;
    static constexpr int XS = XT == APMS_GRAD_F32 ? 4 : 2, HS = HT == APMS_GRAD_F32 ? 4 : 2;
    static constexpr int P_DY = NU * L::E * XS / 16, P_H = NU * L::E * HS / 16, PIECES = P_DY + 2 * P_H;
    static constexpr int STAGES = !VECTOR ? 3 : PIECES <= 6 ? 4 : PIECES <= 8 ? 3 : PIECES <= 12 ? 2 : 1;      // at most 400 bytes a thread
};

template <int XT, int HT, int WT, bool CARRY, bool VECTOR, int NU, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
k_rms_back_team(const RmsBackArgs a, int team_warps, int dy_room, int h_room)
{
    using S = BackShape<XT, HT, VECTOR, NU>;
    using L = typename S::L;
    constexpr int E = L::E, H = E / 2, STAGES = S::STAGES, PIECE = 16 * THREADS, XS = S::XS, HS = S::HS, DX = E * XS / 16, DH = E * HS / 16;
    extern __shared__ __align__(16) char ring[];
    __shared__ float red[2][kTeamWarps];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp / team_warps, unit0 = (warp - team * team_warps) * NU;
    const int teams = THREADS / 32 / team_warps, width = (int)a.width, c0 = L::column(unit0, lane, 0);
    const bool spare = team >= teams;                // warps behind the last whole team
    const int own = spare ? 0 : width, t = threadIdx.x - team * team_warps * 32;
    const int stage_bytes = VECTOR ? S::PIECES * PIECE : teams * (dy_room + 2 * h_room);
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    char* const room = ring + team * (dy_room + 2 * h_room);
    const int64_t step = (int64_t)gridDim.x * teams, row0 = (int64_t)blockIdx.x * teams;

    // The next row to fetch, and where its operands begin.
    int64_t ahead = spare ? a.rows : row0 + team;
    const char* f_dy = static_cast<const char*>(a.dy) + ahead * a.dy_stride * XS + (VECTOR ? c0 * XS : 0);
    const char* f_h = static_cast<const char*>(a.h) + ahead * a.h_stride * HS + (VECTOR ? c0 * HS : 0);
    const char* f_dh = static_cast<const char*>(a.dh) + ahead * a.dh_stride * HS + (VECTOR ? c0 * HS : 0);
    auto fetch = [&](int stage) {
        if (ahead < a.rows) {
            if (VECTOR) {
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    if (c0 + u * L::UNIT >= width) continue;
                    const uint32_t to = mine + stage * stage_bytes;
#pragma unroll
                    for (int k = 0; k < DX; ++k) copy16_async(to + (u * DX + k) * PIECE, f_dy + u * (L::UNIT * XS) + 16 * k);
#pragma unroll
                    for (int k = 0; k < DH; ++k) copy16_async(to + (S::P_DY + u * DH + k) * PIECE, f_h + u * (L::UNIT * HS) + 16 * k);
                    if (CARRY) {
#pragma unroll
                        for (int k = 0; k < DH; ++k) copy16_async(to + (S::P_DY + S::P_H + u * DH + k) * PIECE, f_dh + u * (L::UNIT * HS) + 16 * k);
                    }
                }
            } else {
                char* to = room + stage * stage_bytes;
                stage_shifted<XS>(to, f_dy, width, t, team_warps * 32);
                stage_shifted<HS>(to + dy_room, f_h, width, t, team_warps * 32);
                if (CARRY) stage_shifted<HS>(to + dy_room + h_room, f_dh, width, t, team_warps * 32);
            }
        }
        commit_copies();
        ahead += step;
        f_dy += step * a.dy_stride * XS;
        f_h += step * a.h_stride * HS;
        if (CARRY) f_dh += step * a.dh_stride * HS;
    };
    // E elements of one operand of a unit: TYPE, `piece` its first piece of the thread (VECTOR), or the room and the row's address
    auto operand = [&](auto type, float2* f, int stage, int piece, int room_at, const char* row, int u) {
        constexpr int TYPE = decltype(type)::value, WORDS = E * (TYPE == APMS_GRAD_F32 ? 4 : 2) / 4;
        if (VECTOR) {
            uint32_t w[WORDS];
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) load_shared16(w + k, mine + stage * stage_bytes + (piece + u * (WORDS / 4) + k / 4) * PIECE);
            unpack_words<TYPE, WORDS>(f, w);
        } else {
            constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2;
            const uint32_t from = (uint32_t)__cvta_generic_to_shared(room) + stage * stage_bytes + room_at + (uint32_t)((uintptr_t)row & 15) + c0 * ES;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float v = u * L::UNIT + 32 * j < own - c0 ? load_shared_element<TYPE>(from + (u * L::UNIT + 32 * j) * ES) : 0.0f;
                if (j & 1) f[j / 2].y = v; else f[j / 2].x = v;
            }
        }
    };
    using TypeX = std::integral_constant<int, XT>;
    using TypeH = std::integral_constant<int, HT>;

    float2 w[NU][H], dw[NU][H];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        load_unit<WT, L, VECTOR>(w[u], static_cast<const char*>(a.w), unit0 + u, lane, own);
#pragma unroll
        for (int j = 0; j < H; ++j) dw[u][j] = both(0.0f);
    }
    if (VECTOR && c0 + (NU - 1) * L::UNIT >= own)    // where nothing is ever copied there are zeros for good
        for (int u = 0; u < NU; ++u)
            for (int s = 0; s < STAGES && c0 + u * L::UNIT >= own; ++s) {
                for (int k = 0; k < DX; ++k) put_zeros(mine + s * stage_bytes + (u * DX + k) * PIECE);
                for (int k = 0; k < DH; ++k) {
                    put_zeros(mine + s * stage_bytes + (S::P_DY + u * DH + k) * PIECE);
                    put_zeros(mine + s * stage_bytes + (S::P_DY + S::P_H + u * DH + k) * PIECE);
                }
            }
    int64_t row = ahead;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(s);
    float rstd = row < a.rows ? a.rstd[row] : 0.0f;
    int stage = 0, free_stage = STAGES - 1, flip = 0;
    for (int64_t base = row0; base < a.rows; base += step, row += step) {        // the same number of rounds for all of the CTA's teams
        const bool here = row < a.rows;
        const float next_rstd = row + step < a.rows ? a.rstd[row + step] : 0.0f;
        if (VECTOR) {
            fetch(STAGES == 1 ? 0 : free_stage);
            wait_for_copies<STAGES - 1>();
        } else {                                     // the row is whole once every thread's copies are; the stage behind it has been read by then
            wait_for_copies<STAGES - 2 < 0 ? 0 : STAGES - 2>();
            __syncthreads();
            fetch(free_stage);
        }
        const char* dyr = static_cast<const char*>(a.dy) + row * a.dy_stride * XS;
        const char* hr = static_cast<const char*>(a.h) + row * a.h_stride * HS;
        float2 dy[NU][H], xh[NU][H];
        float2 acc = both(0.0f);
        if (here) {
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                operand(TypeX(), dy[u], stage, 0, 0, dyr, u);
                operand(TypeH(), xh[u], stage, S::P_DY, dy_room, hr, u);
#pragma unroll
                for (int j = 0; j < H; ++j) {
                    xh[u][j] = mul2(xh[u][j], both(rstd));
                    dw[u][j] = fma2(dy[u][j], xh[u][j], dw[u][j]);
                    dy[u][j] = mul2(w[u][j], dy[u][j]);                // a = w dy from here on
                    acc = fma2(dy[u][j], xh[u][j], acc);
                }
            }
        }
        float mean = warp_total(acc.x + acc.y);
        if (team_warps > 1) {
            if (lane == 0) red[flip][warp] = mean;
            __syncthreads();
            const float* sums = red[flip] + (spare ? 0 : team * team_warps);
            mean = sums[0];
            for (int k = 1; k < team_warps; ++k) mean += sums[k];
            flip ^= 1;                                                 // one barrier a sum: the next row's go elsewhere
        }
        if (here) {
            const float2 minus = both(-mean * a.inv_width), by = both(rstd);
            char* dxp = static_cast<char*>(a.dx) + row * width * XS;
            char* drp = static_cast<char*>(a.dr) + row * width * HS;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                float2 dh[H];
                if (CARRY) operand(TypeH(), dh, stage, S::P_DY + S::P_H, dy_room + h_room, static_cast<const char*>(a.dh) + row * a.dh_stride * HS, u);
#pragma unroll
                for (int j = 0; j < H; ++j) {
                    const float2 inner = fma2(xh[u][j], minus, dy[u][j]);
                    dy[u][j] = CARRY ? fma2(inner, by, dh[j]) : mul2(inner, by);
                }
                store_unit<XT, L, VECTOR>(dxp, dy[u], unit0 + u, lane, width);
                if (a.dr) store_unit<HT, L, VECTOR>(drp, dy[u], unit0 + u, lane, width);
            }
        }
        rstd = next_rstd;
        free_stage = stage;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }

    // the CTA's shares: its teams' in order
    wait_for_copies<0>();
    __syncthreads();
    float* shares = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int c = L::column(unit0 + u, lane, j);
            if (c < own) shares[team * width + c] = j & 1 ? dw[u][j / 2].y : dw[u][j / 2].x;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += THREADS) {
        float s = shares[c];
        for (int k = 1; k < teams; ++k) s += shares[k * width + c];
        a.partial[(int64_t)blockIdx.x * width + c] = s;
    }
}

// dweight from the CTAs' shares: 32 columns a CTA, each of its 32 warps a strip of the shares, the strips in order.
__global__ void __launch_bounds__(1024)
k_rms_back_shares(const RmsBackArgs a, int count)
{
    __shared__ float strips[32][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const int strip = threadIdx.x >> 5;
    wait_for_last_kernel();
    float acc = 0.0f;
    if (c < a.width) {
#pragma unroll 4
        for (int k = strip; k < count; k += 32) acc += a.partial[k * a.width + c];
    }
    strips[strip][threadIdx.x & 31] = acc;
    __syncthreads();
    if (strip == 0 && c < a.width) {
        for (int k = 1; k < 32; ++k) acc += strips[k][threadIdx.x & 31];
        store_element(a.dw, c, a.w_type, acc);
    }
}

// Rows wider than a team's registers hold (16,384), or off the 16-byte boundary and wider than three stages of dy, h and dh in shared memory
// (12,504 in 16 bits, 7504 with a binary32 stream, 6252 in binary32): read twice, once for dx and once for dweight.
__global__ void __launch_bounds__(kRmsThreads)
k_rms_back_rows(const RmsBackArgs a)
{
    __shared__ double red[kRmsThreads / 32];
    const int64_t row = blockIdx.x;
    const float rstd = a.rstd[row];
    double acc = 0.0;                                // as in k_rms_rows: the chain is up to 65,536 long
    for (int64_t c = threadIdx.x; c < a.width; c += kRmsThreads) {
        const float xh = load_element(a.h, row * a.h_stride + c, a.h_type) * rstd;
        acc = fma((double)(load_element(a.w, c, a.w_type) * load_element(a.dy, row * a.dy_stride + c, a.dy_type)), (double)xh, acc);
    }
    const float mean = (float)(block_total(acc, red) / (double)a.width);
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

// Teams of warps for rows of `units` units: as few warps as hold them, NU units each; several rows a CTA where that leaves it below
// 128 threads.  0 threads: the rows are too wide.
struct Team { int warps, threads, rows; };
Team team_for(int64_t units, int nu)
{
    Team t = {(int)((units + nu - 1) / nu), 0, 0};
    if (t.warps > kTeamWarps) return t;
    t.rows = t.warps >= 4 ? 1 : 4 / t.warps;
    t.threads = t.warps * t.rows * 32;
    return t;
}

// The kernel of a shape; false: too wide for it.  Elements a lane: so many that about eight 16-byte pieces of x and residual are in flight
// (bfloat16 with a residual at 16 / 32 / 64 elements: 45.7 / 44.5 / 51 us on 8192x4096, binary32 at 16 / 32: 82.6 / 84.0 us).
template <int XT, int RT, int WT>
struct RmsLaunch {
    static constexpr int XS = XT == APMS_GRAD_F32 ? 4 : 2, RS = RT == APMS_GRAD_F32 ? 4 : 2;

    template <int TL>
    static cudaError_t narrow(const RmsArgs& a, int64_t rows, cudaStream_t stream)
    {
        const int64_t each = 128 / TL * 4;
        return launch(k_rms_narrow<XT, RT, WT, TL>, dim3((unsigned)((rows + each - 1) / each)), 128, 0, stream, false, a, rows);
    }

    template <int NU>
    static bool staged(const RmsArgs& a, int64_t rows, int units, cudaStream_t stream, cudaError_t* e)
    {
        const Team t = team_for(units, NU);
        const dim3 block(t.warps * 32, t.rows);
        const size_t x_bytes = (size_t)t.threads * NU * 16, grid = (rows + t.rows - 1) / std::max(1, t.rows);
        if (!t.threads) return false;
        if constexpr (RT == XT) {                    // without a residual its type is x's
            if (!a.r) return with_shared<k_rms_staged<XT, RT, WT, false, NU>>(block, grid, x_bytes, stream, e, a, rows);
        }
        return with_shared<k_rms_staged<XT, RT, WT, true, NU>>(block, grid, x_bytes * (1 + RS / XS), stream, e, a, rows);
    }

    template <int NU>
    static bool shifted(const RmsArgs& a, int64_t rows, int units, cudaStream_t stream, cudaError_t* e)
    {
        const Team t = team_for(units, NU);
        if (!t.threads) return false;
        const int padded = t.warps * NU * 128, x_room = padded * XS + 16, r_room = a.r ? padded * RS + 16 : 0;
        const dim3 block(t.warps * 32, t.rows);
        const size_t grid = (rows + t.rows - 1) / t.rows, shared = (size_t)t.rows * (x_room + r_room);
        if constexpr (RT == XT) {
            if (!a.r) return with_shared<k_rms_shifted<XT, RT, WT, false, NU>>(block, grid, shared, stream, e, a, rows, x_room, r_room);
        }
        return with_shared<k_rms_shifted<XT, RT, WT, true, NU>>(block, grid, shared, stream, e, a, rows, x_room, r_room);
    }

    // KERNEL with as much shared memory as it asks for, within what a CTA can have
    template <auto KERNEL, class... Args>
    static bool with_shared(dim3 block, int64_t grid, size_t shared, cudaStream_t stream, cudaError_t* e, const Args&... args)
    {
        static Resident resident[kMostDevices];
        int ctas = 0;
        if (shared > kMostShared) return false;
        *e = resident_ctas(resident, reinterpret_cast<const void*>(KERNEL), kTeamWarps * 32, kMostShared, &ctas);
        if (*e == cudaSuccess) *e = launch(KERNEL, dim3((unsigned)grid), block, shared, stream, false, args...);
        return true;
    }

    static bool rows(const RmsArgs& a, int64_t rows, bool vector, cudaStream_t stream, cudaError_t* e)
    {
        if (!vector) {
            const int units = (int)((a.width + 127) / 128);
            return units == 1 ? shifted<1>(a, rows, units, stream, e) : units == 2 ? shifted<2>(a, rows, units, stream, e)
                 : shifted<4>(a, rows, units, stream, e) || shifted<8>(a, rows, units, stream, e) || shifted<16>(a, rows, units, stream, e);
        }
        using L = Lanes<XT, true>;
        const int lanes = (int)((a.width + L::E - 1) / L::E), units = (lanes + 31) / 32;
        if (lanes <= 32) {
            *e = lanes <= 8 ? narrow<8>(a, rows, stream) : lanes <= 16 ? narrow<16>(a, rows, stream) : narrow<32>(a, rows, stream);
            return true;
        }
        if (units == 2) return staged<2>(a, rows, units, stream, e);
        return staged<4>(a, rows, units, stream, e) || staged<8>(a, rows, units, stream, e) || staged<16>(a, rows, units, stream, e);
    }
};

template <int XT, int RT>
bool launch_rows(const RmsArgs& a, int64_t rows, bool vector, cudaStream_t stream, cudaError_t* e)
{
    return a.w_type == XT ? RmsLaunch<XT, RT, XT>::rows(a, rows, vector, stream, e) : RmsLaunch<XT, RT, APMS_GRAD_F32>::rows(a, rows, vector, stream, e);
}

bool launch_rms(const RmsArgs& a, int64_t rows, bool vector, cudaStream_t stream, cudaError_t* e)
{
    const bool wide = a.r && a.r_type == APMS_GRAD_F32;
    if (a.x_type == APMS_GRAD_F32) return launch_rows<APMS_GRAD_F32, APMS_GRAD_F32>(a, rows, vector, stream, e);
    if (a.x_type == APMS_GRAD_BF16) return wide ? launch_rows<APMS_GRAD_BF16, APMS_GRAD_F32>(a, rows, vector, stream, e) : launch_rows<APMS_GRAD_BF16, APMS_GRAD_BF16>(a, rows, vector, stream, e);
    return wide ? launch_rows<APMS_GRAD_F16, APMS_GRAD_F32>(a, rows, vector, stream, e) : launch_rows<APMS_GRAD_F16, APMS_GRAD_F16>(a, rows, vector, stream, e);
}

constexpr int kMostShares = 512;

template <int XT, int HT, int WT, bool CARRY, bool VECTOR, int NU, int THREADS>
bool launch_back(const RmsBackArgs& a, int team_warps, cudaStream_t stream, cudaError_t* e)
{
    using S = BackShape<XT, HT, VECTOR, NU>;
    const int teams = THREADS / 32 / team_warps;
    const int dy_room = (int)((a.width * S::XS + 15 + 15) / 16 * 16), h_room = (int)((a.width * S::HS + 15 + 15) / 16 * 16);
    const size_t operands = VECTOR ? (size_t)S::STAGES * S::PIECES * 16 * THREADS : (size_t)S::STAGES * teams * (dy_room + 2 * h_room);
    const size_t shared = std::max(operands, (size_t)teams * a.width * sizeof(float));         // the ring, then the teams' shares
    if (shared > kMostShared) return false;
    auto kernel = k_rms_back_team<XT, HT, WT, CARRY, VECTOR, NU, THREADS>;
    static Resident resident[kMostDevices];          // asked once per kernel and device
    int ctas = 0;
    *e = resident_ctas(resident, reinterpret_cast<const void*>(kernel), THREADS, VECTOR ? shared : kMostShared / (512 / THREADS), &ctas);
    if (*e != cudaSuccess) return true;
    if (!VECTOR) *e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared);
    const int grid = (int)std::min<int64_t>((a.rows + teams - 1) / teams, std::min(kMostShares, ctas));
    if (*e == cudaSuccess) *e = launch(kernel, dim3((unsigned)grid), THREADS, shared, stream, false, a, team_warps, dy_room, h_room);
    if (*e == cudaSuccess) *e = launch(k_rms_back_shares, dim3((unsigned)((a.width + 31) / 32)), 1024, 0, stream, true, a, grid);
    return true;
}

// Lane elements: 16 for rows that 8 warps hold so, then 16 warps with 16 and with 32; 8 for the narrowest rows.
template <int XT, int HT, int WT, bool CARRY, bool VECTOR>
bool launch_back_width(const RmsBackArgs& a, cudaStream_t stream, cudaError_t* e)
{
    using L = Lanes<XT, VECTOR>;
    constexpr int N8 = 8 / L::E, N16 = 16 / L::E, N32 = 32 / L::E;
    const int64_t warps8 = (a.width + 32 * 8 - 1) / (32 * 8), warps16 = (a.width + 32 * 16 - 1) / (32 * 16), warps32 = (a.width + 32 * 32 - 1) / (32 * 32);
    if (warps8 == 1) return launch_back<XT, HT, WT, CARRY, VECTOR, N8, 256>(a, 1, stream, e);
    if (warps16 <= 8 && launch_back<XT, HT, WT, CARRY, VECTOR, N16, 256>(a, (int)warps16, stream, e)) return true;
    if (warps16 <= 16 && launch_back<XT, HT, WT, CARRY, VECTOR, N16, 512>(a, (int)warps16, stream, e)) return true;
    // wider than 8192: three rows off the boundary fit into shared memory in 16 bits only
    constexpr int XS = XT == APMS_GRAD_F32 ? 4 : 2, HS = HT == APMS_GRAD_F32 ? 4 : 2;
    if constexpr (VECTOR || (size_t)BackShape<XT, HT, VECTOR, N32>::STAGES * (XS + 2 * HS) * 8192 <= kMostShared)
        return warps32 <= 16 && launch_back<XT, HT, WT, CARRY, VECTOR, N32, 512>(a, (int)warps32, stream, e);
    return false;
}

template <int XT, int HT, int WT>
bool launch_back_rows(const RmsBackArgs& a, bool vector, cudaStream_t stream, cudaError_t* e)
{
    if (a.dh) return vector ? launch_back_width<XT, HT, WT, true, true>(a, stream, e) : launch_back_width<XT, HT, WT, true, false>(a, stream, e);
    return vector ? launch_back_width<XT, HT, WT, false, true>(a, stream, e) : launch_back_width<XT, HT, WT, false, false>(a, stream, e);
}

template <int XT>
bool launch_back_types(const RmsBackArgs& a, bool vector, cudaStream_t stream, cudaError_t* e)
{
    if (a.h_type == XT) return a.w_type == XT ? launch_back_rows<XT, XT, XT>(a, vector, stream, e) : launch_back_rows<XT, XT, APMS_GRAD_F32>(a, vector, stream, e);
    return a.w_type == XT ? launch_back_rows<XT, APMS_GRAD_F32, XT>(a, vector, stream, e) : launch_back_rows<XT, APMS_GRAD_F32, APMS_GRAD_F32>(a, vector, stream, e);
}

bool launch_rms_back(const RmsBackArgs& a, bool vector, cudaStream_t stream, cudaError_t* e)
{
    if (a.dy_type == APMS_GRAD_F32) return launch_back_rows<APMS_GRAD_F32, APMS_GRAD_F32, APMS_GRAD_F32>(a, vector, stream, e);
    if (a.dy_type == APMS_GRAD_BF16) return launch_back_types<APMS_GRAD_BF16>(a, vector, stream, e);
    return launch_back_types<APMS_GRAD_F16>(a, vector, stream, e);
}

// Every row begins on a 16-byte boundary and holds whole 16-byte pieces.
bool rows_of_16(const void* p, int64_t stride, int64_t width, int type)
{
    const int64_t es = (int64_t)element_size(type);
    return !p || (((uintptr_t)p & 15u) == 0 && stride * es % 16 == 0 && width * es % 16 == 0);
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
    a.x_type = g.x_type; a.r_type = g.residual_type; a.w_type = g.weight_type; a.eps = g.eps; a.inv_width = 1.0f / (float)g.width;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const bool vector = rows_of_16(a.x, a.x_stride, a.width, a.x_type) && rows_of_16(a.r, a.r_stride, a.width, a.r_type) && rows_of_16(a.w, 0, a.width, a.x_type) &&
                        rows_of_16(a.h, a.width, a.width, a.x_type) && (a.scales ? ((uintptr_t)a.y & 7u) == 0 && a.width % 8 == 0 : rows_of_16(a.y, a.width, a.width, a.x_type));
    cudaError_t e = cudaSuccess;
    if (!launch_rms(a, g.rows, vector, stream, &e))
        e = launch(k_rms_rows, dim3((unsigned)g.rows), kRmsThreads, 0, stream, false, a);
    OPERATOR_CUDA("apms_rms_norm", e);
    return APMS_OK;
}

size_t apms_rms_norm_backward_workspace_bytes(int64_t rows, int64_t width)
{
    if (rows < 0 || rows > kMostRows || width < 1 || width > kMostWidth) return 0;
    return (size_t)std::max<int64_t>(kStrips, std::min<int64_t>(rows, kMostShares)) * (size_t)width * sizeof(float);
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
    a.dy_type = g.dy_type; a.h_type = g.h_type; a.w_type = g.weight_type; a.inv_width = 1.0f / (float)g.width;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    const bool vector = rows_of_16(a.dy, a.dy_stride, a.width, a.dy_type) && rows_of_16(a.h, a.h_stride, a.width, a.dy_type) && rows_of_16(a.dh, a.dh_stride, a.width, a.dy_type) &&
                        rows_of_16(a.w, 0, a.width, a.dy_type) && rows_of_16(a.dx, a.width, a.width, a.dy_type) && rows_of_16(a.dr, a.width, a.width, a.dy_type);
    if (!g.rows) {
        e = launch(k_rms_back_shares, dim3((unsigned)((a.width + 31) / 32)), 1024, 0, stream, false, a, 0);
    } else if (!launch_rms_back(a, vector, stream, &e)) {
        e = launch(k_rms_back_rows, dim3((unsigned)g.rows), kRmsThreads, 0, stream, false, a);
        const unsigned columns = (unsigned)((g.width + kRmsThreads - 1) / kRmsThreads);
        if (e == cudaSuccess) e = launch(k_rms_back_weight, dim3(columns, kStrips), kRmsThreads, 0, stream, false, a);
        if (e == cudaSuccess) e = launch(k_rms_back_shares, dim3((unsigned)((a.width + 31) / 32)), 1024, 0, stream, false, a, kStrips);
    }
    OPERATOR_CUDA("apms_rms_norm_backward", e);
    return APMS_OK;
}

}  // extern "C"
