// Dropout with a mask that is never stored.
// Part of libapms.so: included by layers.cu.
#pragma once

namespace {

struct DropArgs {
    int64_t rows, width, x_stride, r_stride, numel;
    const void *x, *r;
    void* h;
    const long long* rng;
    long long* used;
    uint32_t site, border;
    float scale;
};

// One block of Philox 4x32 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011) with 7 rounds, the fewest that pass
// the whole of the test battery used there.  Its 128 bits are eight 16-bit fractions, so p counts in steps of 2^-16, and the scale is of the p so rounded.  The integer multiplications
// are what costs: 16384 x 4096 bfloat16 without a residual takes 48 us; with 10 rounds 53; with a word an element (p to 2^-32) 59, with 10 rounds 74.
constexpr int kPhiloxRounds = 7;
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < kPhiloxRounds; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

struct Source {
    uint32_t k0, k1, s0, s1, site;
    __device__ __forceinline__ explicit Source(const DropArgs& a)
    {
        const long long seed = a.rng[0], step = a.rng[1];
        k0 = (uint32_t)seed; k1 = (uint32_t)((unsigned long long)seed >> 32);
        s0 = (uint32_t)step; s1 = (uint32_t)((unsigned long long)step >> 32);
        site = a.site;
        if (blockIdx.x == 0 && threadIdx.x == 0 && a.used) { a.used[0] = seed; a.used[1] = step; }
    }
    __device__ __forceinline__ uint4 eight(uint32_t number) const { return philox(make_uint4(number, site, s0, s1), k0, k1); }
};

__device__ __forceinline__ float dropped(float x, uint32_t bits, const DropArgs& a) { return bits >= a.border ? x * a.scale : 0.0f; }

// Rows of whole groups of eight that load8 can read (contiguous tensors: one row of any length): UNITS groups a thread, all loaded first.
// Bound by HBM: 16384 x 4096 bfloat16 with a residual 62 us, the rate of a copy; without one 48 us, 0.87 of it.
template <int XT, int RT, bool RESIDUAL, int HT, int UNITS>
__global__ void __launch_bounds__(256) k_dropout(DropArgs a)
{
    const int64_t units = a.numel / 8, first = (int64_t)blockIdx.x * (256 * UNITS) + threadIdx.x, per_row = a.width / 8;
    Eight<XT> x[UNITS];
    Eight<RT> r[RESIDUAL ? UNITS : 1];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const int64_t u = first + k * 256;
        if (u >= units) break;
        int64_t row = 0, col = u * 8;
        if (a.rows > 1) { row = units <= 0xffffffffll ? (uint32_t)u / (uint32_t)per_row : u / per_row; col = (u - row * per_row) * 8; }
        x[k] = load8<XT>(a.x, row * a.x_stride + col);
        if (RESIDUAL) r[k] = load8<RT>(a.r, row * a.r_stride + col);
    }
    const Source source(a);
    if (blockIdx.x == 0 && threadIdx.x < (a.numel & 7)) {                      // one row's last elements
        const int64_t i = units * 8 + threadIdx.x;
        const uint4 bits = source.eight((uint32_t)units);
        const uint32_t word = threadIdx.x < 4 ? threadIdx.x < 2 ? bits.x : bits.y : threadIdx.x < 6 ? bits.z : bits.w;
        const float v = dropped(load1<XT>(a.x, i), threadIdx.x & 1 ? word >> 16 : word & 0xffffu, a);
        store1<HT>(a.h, i, RESIDUAL ? v + load1<RT>(a.r, i) : v);
    }
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const int64_t u = first + k * 256;
        if (u >= units) break;
        const uint4 bits = source.eight((uint32_t)u);
        const uint32_t word[4] = {bits.x, bits.y, bits.z, bits.w};
        float v[8], q[8];
        values8<XT>(v, x[k]);
        if (RESIDUAL) values8<RT>(q, r[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = dropped(v[j], j & 1 ? word[j / 2] >> 16 : word[j / 2] & 0xffffu, a);
            if (RESIDUAL) v[j] += q[j];
        }
        store8<HT>(a.h, u * 8, v);
    }
}

// Any width and alignment: a warp takes kSpans times 256 consecutive elements, whose 32 blocks its lanes form and share, and goes over them 64 at a time, two a lane.  FLAT: one row.
// Bound by the instructions (31 an element): 7777 x 1001 binary32 into bfloat16 12.3 us, 3.8 TB/s.
constexpr int kSpans = 2;
template <int XT, int RT, bool RESIDUAL, int HT, bool FLAT>
__global__ void __launch_bounds__(256) k_dropout_any(DropArgs a, int pairs)
{
    __shared__ uint4 words[8][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t span = ((int64_t)blockIdx.x * 8 + warp) * (256 * kSpans), first = span + lane * 2;
    if (span >= a.numel) return;
    const int width = FLAT ? 0 : (int)a.width;
    const int64_t row = FLAT ? 0 : a.numel <= 0xffffffffll ? (uint32_t)first / (uint32_t)width : first / width;
    int col = FLAT ? 0 : (int)(first - row * width);
    const auto* px = static_cast<const typename Element<XT>::T*>(a.x) + (FLAT ? first : row * a.x_stride + col);
    const auto* pr = static_cast<const typename Element<RT>::T*>(a.r) + (FLAT ? first : row * a.r_stride + col);
    const int64_t x_next = FLAT ? 0 : a.x_stride - width, r_next = FLAT ? 0 : a.r_stride - width;        // from a row's end to the next one's beginning
    auto* h = static_cast<typename Element<HT>::T*>(a.h) + first;
    const uint32_t* bits = reinterpret_cast<const uint32_t*>(words[warp]) + lane;
    const Source source(a);

    auto pass = [&](auto whole, int64_t left) {                     // left: elements from this lane's first one on
        float x[4][2], r[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                x[k][j] = r[k][j] = 0.0f;
                const bool next = !FLAT && j && col + 1 == width;   // the second of a pair, in the next row
                if (whole.value || k * 64 + j < left) {
                    x[k][j] = (float)px[next ? x_next + 1 : j];
                    if (RESIDUAL) r[k][j] = (float)pr[next ? r_next + 1 : j];
                }
            }
            px += 64;
            if (RESIDUAL) pr += 64;
            if (!FLAT)
                for (col += 64; col >= width; col -= width) {
                    px += x_next;
                    if (RESIDUAL) pr += r_next;
                }
        }
        words[warp][lane] = source.eight((uint32_t)(span / 8) + lane);          // behind the loads
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = bits[k * 32];
            float v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                v[j] = dropped(x[k][j], j ? w >> 16 : w & 0xffffu, a);
                if (RESIDUAL) v[j] += r[k][j];
            }
            if (pairs && (whole.value || k * 64 + 1 < left)) {
                if constexpr (HT == APMS_GRAD_F32) *reinterpret_cast<float2*>(h + k * 64) = make_float2(v[0], v[1]);
                else *reinterpret_cast<uint32_t*>(h + k * 64) = pack16<HT>(v[0], v[1]);
            } else {
                if (whole.value || k * 64 < left) store1<HT>(h, k * 64, v[0]);
                if (whole.value || k * 64 + 1 < left) store1<HT>(h, k * 64 + 1, v[1]);
            }
        }
        __syncwarp();
        h += 256;
    };
    for (int s = 0; s < kSpans && span < a.numel; ++s) {
        const int64_t left = a.numel - first;
        if (span + 256 <= a.numel) pass(std::true_type(), left); else pass(std::false_type(), left);
        span += 256;
        first += 256;
    }
}

// Four groups a thread hide the loads' latency where there is enough to do (16384 x 4096: 1 group 4 % slower); below that more CTAs do.
template <int XT, int RT, bool RESIDUAL, int HT>
cudaError_t launch_dropout(const DropArgs& a, bool vector, cudaStream_t stream)
{
    if (!vector) {
        const int pairs = (uintptr_t)a.h % (2 * kBytes<HT>) == 0;
        auto kernel = a.rows == 1 ? k_dropout_any<XT, RT, RESIDUAL, HT, true> : k_dropout_any<XT, RT, RESIDUAL, HT, false>;
        return launch(kernel, dim3((unsigned)((a.numel + 2048 * kSpans - 1) / (2048 * kSpans))), 256, 0, stream, false, a, pairs);
    }
    constexpr int MANY = XT == APMS_GRAD_F32 || RT == APMS_GRAD_F32 ? 2 : 4;
    const int64_t units = a.numel / 8;
    if (units < (int64_t)1024 * 256 * MANY) return launch(k_dropout<XT, RT, RESIDUAL, HT, 1>, dim3((unsigned)(units / 256 + 1)), 256, 0, stream, false, a);
    return launch(k_dropout<XT, RT, RESIDUAL, HT, MANY>, dim3((unsigned)((units + 256 * MANY - 1) / (256 * MANY))), 256, 0, stream, false, a);
}

template <int XT>
cudaError_t launch_dropout_types(const DropArgs& a, int h_type, bool vector, cudaStream_t stream)
{
    if (a.r) return h_type == XT ? launch_dropout<XT, XT, true, XT>(a, vector, stream) : launch_dropout<XT, APMS_GRAD_F32, true, APMS_GRAD_F32>(a, vector, stream);
    if (h_type == XT) return launch_dropout<XT, XT, false, XT>(a, vector, stream);
    if constexpr (XT == APMS_GRAD_F32)
        return h_type == APMS_GRAD_BF16 ? launch_dropout<XT, XT, false, APMS_GRAD_BF16>(a, vector, stream) : launch_dropout<XT, XT, false, APMS_GRAD_F16>(a, vector, stream);
    return cudaErrorInvalidValue;
}

}  // namespace

extern "C" apms_status apms_dropout(const apms_dropout_args* args, void* cuda_stream)
{
    const char* who = "apms_dropout";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_dropout_args& g = *args;
    if (g.rows < 0 || g.width < 1 || g.width > APMS_DROPOUT_MAX || g.rows > APMS_DROPOUT_MAX / g.width)
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld rows of %lld: needs rows >= 0, width >= 1 and at most 2^34 elements", who, (long long)g.rows, (long long)g.width);
    if (g.rows > 1 && g.width > 0x7fffff00) return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld rows of %lld: several rows have at most 2^31 - 256 elements each", who, (long long)g.rows, (long long)g.width);
    if (!known_type(g.x_type) || !known_type(g.h_type)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: unknown element type", who);
    if (g.residual ? g.h_type != g.x_type && g.h_type != APMS_GRAD_F32 : g.h_type != g.x_type && g.x_type != APMS_GRAD_F32)
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: h has x's type, or binary32 with a residual, or 16 bits of a binary32 x without one", who);
    if (!(g.p >= 0.0 && g.p <= 1.0)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: p must be in [0, 1], got %g", who, g.p);
    if (g.site < 0 || g.site > 0xffffffffll) return operator_fail(APMS_ERR_INVALID_ARG, "%s: site must be in [0, 2^32), got %lld", who, (long long)g.site);
    if (!g.rng_dev || (uintptr_t)g.rng_dev % 8 || (uintptr_t)g.used_dev % 8) return operator_fail(APMS_ERR_INVALID_ARG, "%s: rng_dev is NULL, or it or used_dev not 8-byte aligned", who);
    if (g.rows && (!g.x || !g.h)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: x or h is NULL", who);
    if (g.rows > 1 && (g.x_stride < 0 || (g.residual && g.residual_stride < 0))) return operator_fail(APMS_ERR_INVALID_ARG, "%s: a stride is below 0", who);
    if (!on_element(g.x, g.x_type) || !on_element(g.h, g.h_type) || !on_element(g.residual, g.h_type)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (!g.rows) {
        if (g.used_dev) OPERATOR_CUDA("apms_dropout", cudaMemcpyAsync(g.used_dev, g.rng_dev, 16, cudaMemcpyDeviceToDevice, stream));
        return APMS_OK;
    }
    DropArgs a = {};
    a.rows = g.rows; a.width = g.width; a.x_stride = g.x_stride; a.r_stride = g.residual_stride; a.numel = g.rows * g.width;
    a.x = g.x; a.r = g.residual; a.h = g.h; a.rng = (const long long*)g.rng_dev; a.used = (long long*)g.used_dev; a.site = (uint32_t)g.site;
    a.border = (uint32_t)floor(g.p * 65536.0 + 0.5);
    a.scale = a.border < 65536u ? (float)(65536.0 / (65536.0 - a.border)) : 0.0f;
    if (a.rows > 1 && a.x_stride == a.width && (!a.r || a.r_stride == a.width)) { a.width = a.numel; a.rows = 1; }
    const bool vector = on_eight(a.h, g.h_type) && (a.rows == 1 ? on_eight(a.x, g.x_type) && on_eight(a.r, g.h_type) : rows_of_eight(a.x, a.rows, a.x_stride, a.width, g.x_type) && rows_of_eight(a.r, a.rows, a.r_stride, a.width, g.h_type));
    const cudaError_t e = g.x_type == APMS_GRAD_F32 ? launch_dropout_types<APMS_GRAD_F32>(a, g.h_type, vector, stream)
                        : g.x_type == APMS_GRAD_BF16 ? launch_dropout_types<APMS_GRAD_BF16>(a, g.h_type, vector, stream) : launch_dropout_types<APMS_GRAD_F16>(a, g.h_type, vector, stream);
    OPERATOR_CUDA("apms_dropout", e);
    return APMS_OK;
}
