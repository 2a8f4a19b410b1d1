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

// E elements of type TYPE from column `unit`, 0 behind the width.
template <int TYPE, class L, bool VECTOR>
__device__ __forceinline__ void load_unit(float* f, const char* row, int unit, int lane, int width)
{
    constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2;
    if (VECTOR) {
        const int c = L::column(unit, lane, 0);
        uint32_t w[L::E * ES / 4];
        if (c < width) {
#pragma unroll
            for (int k = 0; k < L::E * ES / 4; k += 4) load16(w + k, row + (int64_t)c * ES + 4 * k);
        } else {
#pragma unroll
            for (int k = 0; k < L::E * ES / 4; ++k) w[k] = 0;
        }
#pragma unroll
        for (int k = 0; k < L::E * ES / 4; ++k) {
            if (ES == 4) f[k] = __uint_as_float(w[k]);
            else { const float2 v = unpack16<TYPE>(w[k]); f[(2 * k) % L::E] = v.x; f[(2 * k + 1) % L::E] = v.y; }
        }
    } else {
#pragma unroll
        for (int j = 0; j < L::E; ++j) {
            const int c = L::column(unit, lane, j);
            f[j] = c < width ? load_element(row, c, TYPE) : 0.0f;
        }
    }
}

template <int TYPE, class L, bool VECTOR>
__device__ __forceinline__ void store_unit(char* row, const float* f, int unit, int lane, int width)
{
    constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2;
    if (VECTOR) {
        const int c = L::column(unit, lane, 0);
        if (c >= width) return;
        uint32_t w[L::E * ES / 4];
#pragma unroll
        for (int k = 0; k < L::E * ES / 4; ++k)
            w[k] = ES == 4 ? __float_as_uint(f[k]) : pack16<TYPE == APMS_GRAD_F32 ? APMS_GRAD_BF16 : TYPE>(f[(2 * k) % L::E], f[(2 * k + 1) % L::E]);
#pragma unroll
        for (int k = 0; k < L::E * ES / 4; k += 4) *reinterpret_cast<uint4*>(row + (int64_t)c * ES + 4 * k) = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < L::E; ++j) {
            const int c = L::column(unit, lane, j);
            if (c < width) store_element(row, c, TYPE, f[j]);
        }
    }
}

template <class L, bool VECTOR>
__device__ __forceinline__ void store_unit_e4m3(uint8_t* row, const float* f, int unit, int lane, int width)
{
    if (VECTOR) {
        const int c = L::column(unit, lane, 0);
        if (c >= width) return;
        uint32_t w[L::E / 4];
#pragma unroll
        for (int k = 0; k < L::E / 4; ++k)
            w[k] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[4 * k], f[4 * k + 1]), __NV_SATFINITE, __NV_E4M3) |
                   (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[4 * k + 2], f[4 * k + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
        if (L::E == 8) *reinterpret_cast<uint2*>(row + c) = make_uint2(w[0], w[L::E / 4 - 1]);
        else *reinterpret_cast<uint32_t*>(row + c) = w[0];
    } else {
#pragma unroll
        for (int j = 0; j < L::E; ++j) {
            const int c = L::column(unit, lane, j);
            if (c < width) row[c] = __nv_cvt_float_to_fp8(f[j], __NV_SATFINITE, __NV_E4M3);
        }
    }
}

constexpr int kTeamWarps = 16;                   // a row's at most: with 32 elements a lane, rows of up to 16,384

// Combines a value of each of a team's warps (a row's); TEAM warps of consecutive index.  smem: one T per warp of the CTA.  Every
// thread of the CTA calls it.
template <class T, class Op>
__device__ __forceinline__ T over_team(T v, T* smem, int team_warps, Op op)
{
    if (team_warps == 1) return v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) smem[warp] = v;
    __syncthreads();
    const int first = warp / team_warps * team_warps;
    v = lane < team_warps ? smem[first + lane] : T(0);
#pragma unroll
    for (int o = kTeamWarps; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A team of `team_warps` warps a row, NU units a warp, the row in registers from the first load to the last store: x, the residual
// and the weight are read once (the weight from L1 or L2 after the first rows), h and y written once.  A CTA ends with its row or rows:
// the loads of the next CTAs cover the latency of this one's sum.
template <int XT, int RT, bool VECTOR, int NU>
__global__ void __launch_bounds__(kTeamWarps * 32)
k_rms_team(const RmsArgs a, int64_t rows, int team_warps)
{
    using L = Lanes<XT, VECTOR>;
    constexpr int XS = XT == APMS_GRAD_F32 ? 4 : 2, RS = RT == APMS_GRAD_F32 ? 4 : 2;
    __shared__ float red[kTeamWarps];
    __shared__ uint32_t red_most[kTeamWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp / team_warps, unit0 = (warp - team * team_warps) * NU;
    const int width = (int)a.width;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / 32 / team_warps) + team;
    const bool here = row < rows;
    const int in = here ? width : 0;                 // a team without a row loads nothing and stays for the barriers
    float h[NU][L::E], w[NU][L::E];
    const char* xr = static_cast<const char*>(a.x) + row * a.x_stride * XS;
#pragma unroll
    for (int u = 0; u < NU; ++u) load_unit<XT, L, VECTOR>(h[u], xr, unit0 + u, lane, in);
    if (a.r) {
        const char* rr = static_cast<const char*>(a.r) + row * a.r_stride * RS;
        float r[NU][L::E];
#pragma unroll
        for (int u = 0; u < NU; ++u) load_unit<RT, L, VECTOR>(r[u], rr, unit0 + u, lane, in);
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < L::E; ++j) h[u][j] += r[u][j];
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        if (a.w_type == APMS_GRAD_F32) load_unit<APMS_GRAD_F32, L, VECTOR>(w[u], static_cast<const char*>(a.w), unit0 + u, lane, in);
        else load_unit<XT, L, VECTOR>(w[u], static_cast<const char*>(a.w), unit0 + u, lane, in);
    }
    float acc = 0.0f;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < L::E; ++j) acc = fmaf(h[u][j], h[u][j], acc);
    if (a.r) {
        char* hr = static_cast<char*>(a.h) + row * a.width * RS;
#pragma unroll
        for (int u = 0; u < NU; ++u) store_unit<RT, L, VECTOR>(hr, h[u], unit0 + u, lane, in);
    }
    acc = over_team(warp_total(acc), red, team_warps, [](float p, float q) { return p + q; });
    const float rstd = __frsqrt_rn(acc / (float)width + a.eps);
    if (here && unit0 == 0 && lane == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < L::E; ++j) h[u][j] = h[u][j] * rstd * w[u][j];
    if (!a.scales) {
        char* yr = static_cast<char*>(a.y) + row * a.width * XS;
#pragma unroll
        for (int u = 0; u < NU; ++u) store_unit<XT, L, VECTOR>(yr, h[u], unit0 + u, lane, in);
        return;
    }
    uint32_t most[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        most[u] = 0;
#pragma unroll
        for (int j = 0; j < L::E; ++j) most[u] = max(most[u], L::column(unit0 + u, lane, j) < in ? magnitude_bits(h[u][j]) : 0u);
    }
    uint8_t* qr = static_cast<uint8_t*>(a.y) + row * a.width;
    if (a.groups > 1 || a.group != a.width) {        // 128 columns: within a warp
#pragma unroll
        for (int u = 0; u < NU; ++u) {
#pragma unroll
            for (int o = L::GROUP_LANES / 2; o > 0; o >>= 1) most[u] = max(most[u], __shfl_xor_sync(0xffffffffu, most[u], o));
            float scale, inverse;
            group_scale(most[u], &scale, &inverse);
            const int c = L::column(unit0 + u, lane, 0);
            if (lane % L::GROUP_LANES == 0 && c < in) a.scales[row * a.groups + c / 128] = scale;
#pragma unroll
            for (int j = 0; j < L::E; ++j) h[u][j] *= inverse;
            store_unit_e4m3<L, VECTOR>(qr, h[u], unit0 + u, lane, in);
        }
    } else {
        uint32_t m = most[0];
#pragma unroll
        for (int u = 1; u < NU; ++u) m = max(m, most[u]);
        m = over_team(__reduce_max_sync(0xffffffffu, m), red_most, team_warps, [](uint32_t p, uint32_t q) { return max(p, q); });
        float scale, inverse;
        group_scale(m, &scale, &inverse);
        if (here && unit0 == 0 && lane == 0) a.scales[row] = scale;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
#pragma unroll
            for (int j = 0; j < L::E; ++j) h[u][j] *= inverse;
            store_unit_e4m3<L, VECTOR>(qr, h[u], unit0 + u, lane, in);
        }
    }
}

// Rows wider than a team's registers hold: one CTA per row, any stride and alignment, read again for each pass.
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

// 16 bytes from global to shared memory without a register; both 16-byte aligned.  A thread copies what it reads itself,
// so its own wait is all the order that is needed.
__device__ __forceinline__ void copy16_async(const char* to_shared, const char* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"((uint32_t)__cvta_generic_to_shared(to_shared)), "l"(from) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_for_copies() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

// E elements of TYPE from the 16-byte pieces at p, `stride` bytes apart.
template <int TYPE, int E>
__device__ __forceinline__ void unpack_pieces(float* f, const char* p, int stride)
{
    constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2;
#pragma unroll
    for (int k = 0; k < E * ES / 16; ++k) {
        const uint4 v = *reinterpret_cast<const uint4*>(p + k * stride);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (ES == 4) f[4 * k + j] = __uint_as_float(w[j]);
            else { const float2 g = unpack16<TYPE>(w[j]); f[(8 * k + 2 * j) % E] = g.x; f[(8 * k + 2 * j + 1) % E] = g.y; }
        }
    }
}

// A CTA walks over rows, a team of warps each, and keeps its columns' share of dweight in registers; `partial` gets one row of shares per CTA.
// The rows' operands come through a ring of STAGES rows in shared memory, each thread copying its own pieces
// ahead (cp.async: neither registers nor a producer), because one row a CTA in flight at a time would not cover HBM's latency.
// Rows that are not whole 16-byte pieces are loaded directly.
template <int XT, int HT, bool VECTOR, int NU>
struct BackShape {
    using L = Lanes<XT, VECTOR>;
    static constexpr int XS = XT == APMS_GRAD_F32 ? 4 : 2, HS = HT == APMS_GRAD_F32 ? 4 : 2;
    static constexpr int P_DY = VECTOR ? NU * L::E * XS / 16 : 0, P_H = VECTOR ? NU * L::E * HS / 16 : 0, PIECES = P_DY + 2 * P_H;
    static constexpr int STAGES = PIECES <= 6 ? 4 : PIECES <= 8 ? 3 : PIECES <= 12 ? 2 : 1;      // at most 400 bytes a thread
    static constexpr int LANE_ELEMENTS = NU * L::E;
    static constexpr int BYTES_A_THREAD = STAGES * PIECES * 16 > LANE_ELEMENTS * 4 ? STAGES * PIECES * 16 : LANE_ELEMENTS * 4;
};

template <int XT, int HT, bool VECTOR, int NU, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
k_rms_back_team(const RmsBackArgs a, int team_warps)
{
    using S = BackShape<XT, HT, VECTOR, NU>;
    using L = typename S::L;
    constexpr int E = L::E, STAGES = S::STAGES, PIECE = 16 * THREADS;
    extern __shared__ __align__(16) char ring[];
    __shared__ float red[2][2 * kTeamWarps];         // a spare warp looks behind the last team's
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp / team_warps, unit0 = (warp - team * team_warps) * NU;
    const int teams = THREADS / 32 / team_warps, width = (int)a.width;
    const bool spare = team >= teams;                // warps behind the last whole team
    char* mine = ring + threadIdx.x * 16;
    const int64_t step = (int64_t)gridDim.x * teams;
    const int64_t row0 = (int64_t)blockIdx.x * teams, row_mine = spare ? a.rows : row0 + team;

    auto fetch = [&](int64_t row, int stage) {
        if (VECTOR && row < a.rows) {
            char* to = mine + stage * (S::PIECES * PIECE);
            const char* dy = static_cast<const char*>(a.dy) + row * a.dy_stride * S::XS;
            const char* h = static_cast<const char*>(a.h) + row * a.h_stride * S::HS;
            const char* dh = static_cast<const char*>(a.dh) + row * a.dh_stride * S::HS;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const int c = L::column(unit0 + u, lane, 0);
                if (c >= width) continue;
                constexpr int DX = S::P_DY / NU, DH = S::P_H / NU;
#pragma unroll
                for (int k = 0; k < DX; ++k) copy16_async(to + (u * DX + k) * PIECE, dy + (int64_t)c * S::XS + 16 * k);
#pragma unroll
                for (int k = 0; k < DH; ++k) copy16_async(to + (S::P_DY + u * DH + k) * PIECE, h + (int64_t)c * S::HS + 16 * k);
                if (a.dh) {
#pragma unroll
                    for (int k = 0; k < DH; ++k) copy16_async(to + (S::P_DY + S::P_H + u * DH + k) * PIECE, dh + (int64_t)c * S::HS + 16 * k);
                }
            }
        }
        if (VECTOR) commit_copies();
    };

    float w[NU][E], dw[NU][E];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        if (a.w_type == APMS_GRAD_F32) load_unit<APMS_GRAD_F32, L, VECTOR>(w[u], static_cast<const char*>(a.w), unit0 + u, lane, spare ? 0 : width);
        else load_unit<XT, L, VECTOR>(w[u], static_cast<const char*>(a.w), unit0 + u, lane, spare ? 0 : width);
#pragma unroll
        for (int j = 0; j < E; ++j) dw[u][j] = 0.0f;
    }
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(row_mine + s * step, s);
    float rstd = row_mine < a.rows ? a.rstd[row_mine] : 0.0f;
    int stage = 0, flip = 0;
    for (int64_t base = row0; base < a.rows; base += step) {           // the same number of rounds for all of the CTA's teams
        const int64_t row = row_mine + (base - row0);
        const bool here = row < a.rows;
        const int in = here ? width : 0;
        const float next_rstd = row + step < a.rows ? a.rstd[row + step] : 0.0f;
        if (STAGES == 1) fetch(row, 0); else fetch(row + (STAGES - 1) * step, (stage + STAGES - 1) % STAGES);
        if (VECTOR) wait_for_copies<STAGES - 1>();
        const char* from = mine + stage * (S::PIECES * PIECE);
        const char* dyr = static_cast<const char*>(a.dy) + row * a.dy_stride * S::XS;
        const char* hr = static_cast<const char*>(a.h) + row * a.h_stride * S::HS;
        float dy[NU][E], xh[NU][E];
        float acc = 0.0f;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            if (VECTOR) {
                unpack_pieces<XT, E>(dy[u], from + u * (S::P_DY / NU) * PIECE, PIECE);
                unpack_pieces<HT, E>(xh[u], from + (S::P_DY + u * (S::P_H / NU)) * PIECE, PIECE);
                if (L::column(unit0 + u, lane, 0) >= in) {             // nothing was copied there
#pragma unroll
                    for (int j = 0; j < E; ++j) dy[u][j] = xh[u][j] = 0.0f;
                }
            } else {
                load_unit<XT, L, VECTOR>(dy[u], dyr, unit0 + u, lane, in);
                load_unit<HT, L, VECTOR>(xh[u], hr, unit0 + u, lane, in);
            }
#pragma unroll
            for (int j = 0; j < E; ++j) {
                xh[u][j] *= rstd;
                acc = fmaf(w[u][j] * dy[u][j], xh[u][j], acc);
            }
        }
        const float mean = over_team(warp_total(acc), red[flip], team_warps, [](float p, float q) { return p + q; }) / (float)width;
        flip ^= 1;                                                     // one barrier a row: the next row's sums go elsewhere
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float dx[E], dh[E];
            if (a.dh) {
                if (VECTOR) unpack_pieces<HT, E>(dh, from + (S::P_DY + S::P_H + u * (S::P_H / NU)) * PIECE, PIECE);
                else load_unit<HT, L, VECTOR>(dh, static_cast<const char*>(a.dh) + row * a.dh_stride * S::HS, unit0 + u, lane, in);
            }
#pragma unroll
            for (int j = 0; j < E; ++j) {
                dw[u][j] = fmaf(dy[u][j], xh[u][j], dw[u][j]);
                dx[j] = rstd * (w[u][j] * dy[u][j] - xh[u][j] * mean);
                if (a.dh) dx[j] += dh[j];
            }
            store_unit<XT, L, VECTOR>(static_cast<char*>(a.dx) + row * a.width * S::XS, dx, unit0 + u, lane, in);
            if (a.dr) store_unit<HT, L, VECTOR>(static_cast<char*>(a.dr) + row * a.width * S::HS, dx, unit0 + u, lane, in);
        }
        rstd = next_rstd;
        stage = STAGES == 1 ? 0 : (stage + 1) % STAGES;
    }

    // the CTA's shares: its teams' in order
    if (VECTOR) wait_for_copies<0>();
    __syncthreads();
    float* shares = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int c = L::column(unit0 + u, lane, j);
            if (!spare && c < width) shares[team * width + c] = dw[u][j];
        }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += THREADS) {
        float s = shares[c];
        for (int t = 1; t < teams; ++t) s += shares[t * width + c];
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

// Rows wider than a team's registers hold.
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

template <int XT, int RT, bool VECTOR>
bool launch_team(const RmsArgs& a, int64_t rows, cudaStream_t stream, cudaError_t* e)
{
    using L = Lanes<XT, VECTOR>;
    constexpr int MOST = 32 / L::E;                  // 32 elements a lane
    const int64_t units = (a.width + L::UNIT - 1) / L::UNIT;
    const int nu = units == 1 ? 1 : units == 2 ? 2 : MOST;
    const Team t = team_for(units, nu);
    if (!t.threads) return false;
    const dim3 grid((unsigned)((rows + t.rows - 1) / t.rows));
    *e = nu == 1 ? launch(k_rms_team<XT, RT, VECTOR, 1>, grid, t.threads, 0, stream, false, a, rows, t.warps)
       : nu == 2 ? launch(k_rms_team<XT, RT, VECTOR, 2>, grid, t.threads, 0, stream, false, a, rows, t.warps)
                 : launch(k_rms_team<XT, RT, VECTOR, MOST>, grid, t.threads, 0, stream, false, a, rows, t.warps);
    return true;
}

template <bool VECTOR>
bool launch_rows(const RmsArgs& a, int64_t rows, cudaStream_t stream, cudaError_t* e)
{
    const bool wide = a.r && a.r_type == APMS_GRAD_F32;
    if (a.x_type == APMS_GRAD_F32) return launch_team<APMS_GRAD_F32, APMS_GRAD_F32, VECTOR>(a, rows, stream, e);
    if (a.x_type == APMS_GRAD_BF16) return wide ? launch_team<APMS_GRAD_BF16, APMS_GRAD_F32, VECTOR>(a, rows, stream, e) : launch_team<APMS_GRAD_BF16, APMS_GRAD_BF16, VECTOR>(a, rows, stream, e);
    return wide ? launch_team<APMS_GRAD_F16, APMS_GRAD_F32, VECTOR>(a, rows, stream, e) : launch_team<APMS_GRAD_F16, APMS_GRAD_F16, VECTOR>(a, rows, stream, e);
}

constexpr int kMostShares = 512;

template <int XT, int HT, bool VECTOR, int NU, int THREADS>
cudaError_t launch_back(const RmsBackArgs& a, int team_warps, cudaStream_t stream)
{
    using S = BackShape<XT, HT, VECTOR, NU>;
    constexpr size_t shared = (size_t)S::BYTES_A_THREAD * THREADS;
    auto kernel = k_rms_back_team<XT, HT, VECTOR, NU, THREADS>;
    static Resident resident[kMostDevices];          // asked once per kernel and device
    int ctas = 0;
    cudaError_t e = resident_ctas(resident, reinterpret_cast<const void*>(kernel), THREADS, shared, &ctas);
    if (e != cudaSuccess) return e;
    const int teams = THREADS / 32 / team_warps;
    const int grid = (int)std::min<int64_t>((a.rows + teams - 1) / teams, std::min(kMostShares, ctas));
    e = launch(kernel, dim3((unsigned)grid), THREADS, shared, stream, false, a, team_warps);
    if (e != cudaSuccess) return e;
    return launch(k_rms_back_shares, dim3((unsigned)((a.width + 31) / 32)), 1024, 0, stream, true, a, grid);
}

// Lane elements: 16 for rows that 8 warps hold so, then 16 warps with 16 and with 32; 8 for the narrowest rows.
template <int XT, int HT, bool VECTOR>
bool launch_back_width(const RmsBackArgs& a, cudaStream_t stream, cudaError_t* e)
{
    using L = Lanes<XT, VECTOR>;
    constexpr int N8 = 8 / L::E, N16 = 16 / L::E, N32 = 32 / L::E;
    const int64_t warps8 = (a.width + 32 * 8 - 1) / (32 * 8), warps16 = (a.width + 32 * 16 - 1) / (32 * 16), warps32 = (a.width + 32 * 32 - 1) / (32 * 32);
    if (warps8 == 1) *e = launch_back<XT, HT, VECTOR, N8, 256>(a, 1, stream);
    else if (warps16 <= 8) *e = launch_back<XT, HT, VECTOR, N16, 256>(a, (int)warps16, stream);
    else if (warps16 <= 16) *e = launch_back<XT, HT, VECTOR, N16, 512>(a, (int)warps16, stream);
    else if (warps32 <= 16) *e = launch_back<XT, HT, VECTOR, N32, 512>(a, (int)warps32, stream);
    else return false;
    return true;
}

template <bool VECTOR>
bool launch_back_rows(const RmsBackArgs& a, cudaStream_t stream, cudaError_t* e)
{
    const bool wide = a.h_type == APMS_GRAD_F32;
    if (a.dy_type == APMS_GRAD_F32) return launch_back_width<APMS_GRAD_F32, APMS_GRAD_F32, VECTOR>(a, stream, e);
    if (a.dy_type == APMS_GRAD_BF16) return wide ? launch_back_width<APMS_GRAD_BF16, APMS_GRAD_F32, VECTOR>(a, stream, e) : launch_back_width<APMS_GRAD_BF16, APMS_GRAD_BF16, VECTOR>(a, stream, e);
    return wide ? launch_back_width<APMS_GRAD_F16, APMS_GRAD_F32, VECTOR>(a, stream, e) : launch_back_width<APMS_GRAD_F16, APMS_GRAD_F16, VECTOR>(a, stream, e);
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
    a.x_type = g.x_type; a.r_type = g.residual_type; a.w_type = g.weight_type; a.eps = g.eps;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const bool vector = rows_of_16(a.x, a.x_stride, a.width, a.x_type) && rows_of_16(a.r, a.r_stride, a.width, a.r_type) && rows_of_16(a.w, 0, a.width, a.x_type) &&
                        rows_of_16(a.h, a.width, a.width, a.x_type) && (a.scales ? ((uintptr_t)a.y & 7u) == 0 && a.width % 8 == 0 : rows_of_16(a.y, a.width, a.width, a.x_type));
    cudaError_t e = cudaSuccess;
    if (!(vector ? launch_rows<true>(a, g.rows, stream, &e) : launch_rows<false>(a, g.rows, stream, &e)))
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
    a.dy_type = g.dy_type; a.h_type = g.h_type; a.w_type = g.weight_type;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    const bool vector = rows_of_16(a.dy, a.dy_stride, a.width, a.dy_type) && rows_of_16(a.h, a.h_stride, a.width, a.dy_type) && rows_of_16(a.dh, a.dh_stride, a.width, a.dy_type) &&
                        rows_of_16(a.w, 0, a.width, a.dy_type) && rows_of_16(a.dx, a.width, a.width, a.dy_type) && rows_of_16(a.dr, a.width, a.width, a.dy_type);
    if (!g.rows) {
        e = launch(k_rms_back_shares, dim3((unsigned)((a.width + 31) / 32)), 1024, 0, stream, false, a, 0);
    } else if (!(vector ? launch_back_rows<true>(a, stream, &e) : launch_back_rows<false>(a, stream, &e))) {
        e = launch(k_rms_back_rows, dim3((unsigned)g.rows), kRmsThreads, 0, stream, false, a);
        const unsigned columns = (unsigned)((g.width + kRmsThreads - 1) / kRmsThreads);
        if (e == cudaSuccess) e = launch(k_rms_back_weight, dim3(columns, kStrips), kRmsThreads, 0, stream, false, a);
        if (e == cudaSuccess) e = launch(k_rms_back_shares, dim3((unsigned)((a.width + 31) / 32)), 1024, 0, stream, false, a, kStrips);
    }
    OPERATOR_CUDA("apms_rms_norm_backward", e);
    return APMS_OK;
}

}  // extern "C"
