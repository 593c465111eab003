// rowquant.hip -- quantizers with a scale for each row or each column, and the
// transposition of int8 codes: the operands of iseg_matmul_i8.
//
// Every decision is exact: v = x mul is held in double where mul is given
// (24 x 24 bits), the largest magnitude is taken on the bit patterns (where a
// NaN or an infinity is larger than every finite value, so it is seen), and a
// code is settled by the sign of v - (n + 1/2) scale in double, whose product
// is exact (9 x 24 bits).
#include "rowops.h"

namespace {

constexpr float kScaleMin = 1.17549435e-38f;      // 2^-126
constexpr uint64_t kAbs64 = 0x7fffffffffffffffull;
constexpr uint64_t kInf64 = 0x7ff0000000000000ull;

struct RqRowArgs {
    const void* x;
    const float* mul;
    int8_t* codes;
    float *scale, *sums;
    uint64_t* pmax;              // columns: [strips][C] bit patterns of the largest |v|
    float* psum;                 // columns: [strips][C] partial sums of x
    int64_t M, C, x_ld, codes_ld;
    int32_t bits, mode;
    int32_t* status;
};

// scale of a largest magnitude given as a double's bits; NaN if there is none
__device__ __forceinline__ float scale_of(uint64_t big, int bits, int mode)
{
    if (big >= kInf64) return __builtin_nanf("");
    if (big == 0) return 1.f;
    const double t = __builtin_bit_cast(double, big);
    double s;
    if (mode == ISEG_SCALE_POW2) {
        int e;
        (void)frexp(t, &e);                        // t = f 2^e with f in [1/2, 1): 2^e is the power above t
        s = ldexp(1.0, e + 1 - bits);
    } else {
        s = t / (double)((1 << (bits - 1)) - 1);
    }
    const float f = (float)s;
    return f < kScaleMin ? kScaleMin : (f <= 3.4028234e38f ? f : __builtin_nanf(""));
}

// clamp(floor(v / s + 1/2), +-lim): an estimate within one, then the two half-steps around it
__device__ __forceinline__ int code_of(double v, float s, float inv, int lim)
{
    float q = fminf(fmaxf((float)v * inv, -128.f), 128.f);
    int n = (int)floorf(q + 0.5f);
    const double sd = (double)s;
    if (v - ((double)n + 0.5) * sd >= 0.0) n++;
    else if (v - ((double)n - 0.5) * sd < 0.0) n--;
    return n > lim ? lim : (n < -lim ? -lim : n);
}

__device__ __forceinline__ uint64_t bits_of(double v) { return __builtin_bit_cast(uint64_t, v) & kAbs64; }

// ---------------------------------------------------------------------------
// rows: one block per row, the row read twice (the second time from the caches)
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_rows(RqRowArgs a)
{
    const int tid = threadIdx.x;
    const int lim = (1 << (a.bits - 1)) - 1;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        int8_t* o = a.codes + m * a.codes_ld;
        uint64_t big = 0;
        for (int64_t c = tid; c < a.C; c += 256) {
            const double v = a.mul ? (double)(float)x[c] * (double)a.mul[c] : (double)(float)x[c];
            const uint64_t b = bits_of(v);
            big = b > big ? b : big;
        }
        big = block_max_u64(big);
        const float s = scale_of(big, a.bits, a.mode);
        const bool ok = s == s;
        if (tid == 0) {
            a.scale[m] = s;
            if (!ok) set_status(a.status, ISEG_DEV_NONFINITE);
        }
        const float inv = 1.f / s;
        for (int64_t c = tid; c < a.C; c += 256) {
            const double v = a.mul ? (double)(float)x[c] * (double)a.mul[c] : (double)(float)x[c];
            o[c] = ok ? (int8_t)code_of(v, s, inv, lim) : 0;
        }
    }
}

// ---------------------------------------------------------------------------
// columns
// ---------------------------------------------------------------------------
// Largest |v| and sum of x of 64 columns over a strip of rows.
template <typename T>
__global__ __launch_bounds__(256) void k_cols_stats(RqRowArgs a, int64_t strip)
{
    __shared__ uint64_t rm[4][64];
    __shared__ float rs[4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    const int64_t m0 = (int64_t)blockIdx.y * strip;
    const int64_t m1 = m0 + strip < a.M ? m0 + strip : a.M;
    uint64_t big = 0;
    float sum = 0.f;
    if (c < a.C)
        for (int64_t m = m0 + w; m < m1; m += 4) {
            const float x = (float)((const T*)a.x)[m * a.x_ld + c];
            const uint64_t b = bits_of(a.mul ? (double)x * (double)a.mul[m] : (double)x);
            big = b > big ? b : big;
            sum += x;
        }
    rm[w][lane] = big;
    rs[w][lane] = sum;
    __syncthreads();
    if (w != 0 || c >= a.C) return;
    for (int i = 1; i < 4; i++) {
        big = rm[i][lane] > big ? rm[i][lane] : big;
        sum += rs[i][lane];
    }
    a.pmax[(int64_t)blockIdx.y * a.C + c] = big;
    a.psum[(int64_t)blockIdx.y * a.C + c] = sum;
}

__global__ __launch_bounds__(256) void k_cols_scale(RqRowArgs a, int strips)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.C) return;
    uint64_t big = 0;
    float sum = 0.f;
    for (int i = 0; i < strips; i++) {
        const uint64_t b = a.pmax[(int64_t)i * a.C + c];
        big = b > big ? b : big;
        sum += a.psum[(int64_t)i * a.C + c];
    }
    const float s = scale_of(big, a.bits, a.mode);
    a.scale[c] = s;
    if (a.sums) a.sums[c] = sum;
    if (!(s == s)) set_status(a.status, ISEG_DEV_NONFINITE);
}

// codes of a 64 x 64 tile, turned in LDS (rows of 68 bytes: a column of the
// tile then falls on 16 different banks)
template <typename T>
__global__ __launch_bounds__(256) void k_cols_codes(RqRowArgs a)
{
    __shared__ int8_t t[64][68];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int lim = (1 << (a.bits - 1)) - 1;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    const float s = c < a.C ? a.scale[c] : 1.f;
    const bool ok = s == s;
    const float inv = 1.f / s;
    const int64_t mt = ceil_div64(a.M, 64);
    for (int64_t b = blockIdx.y; b < mt; b += gridDim.y) {
        const int64_t m0 = b * 64;
        for (int r = w; r < 64; r += 4) {
            const int64_t m = m0 + r;
            if (m < a.M && c < a.C) {
                const float x = (float)((const T*)a.x)[m * a.x_ld + c];
                const double v = a.mul ? (double)x * (double)a.mul[m] : (double)x;
                t[lane][r] = ok ? (int8_t)code_of(v, s, inv, lim) : 0;
            }
        }
        __syncthreads();
        for (int r = w; r < 64; r += 4) {
            const int64_t cc = (int64_t)blockIdx.x * 64 + r;
            if (cc < a.C && m0 + lane < a.M) a.codes[cc * a.codes_ld + m0 + lane] = t[r][lane];
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void k_transpose_i8(const int8_t* __restrict__ in, int64_t M, int64_t C,
                                                      int64_t in_ld, int8_t* __restrict__ out, int64_t out_ld)
{
    __shared__ int8_t t[64][68];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c0 = (int64_t)blockIdx.x * 64;
    const int64_t mt = ceil_div64(M, 64);
    for (int64_t b = blockIdx.y; b < mt; b += gridDim.y) {
        const int64_t m0 = b * 64;
        for (int r = w; r < 64; r += 4)
            if (m0 + r < M && c0 + lane < C) t[lane][r] = in[(m0 + r) * in_ld + c0 + lane];
        __syncthreads();
        for (int r = w; r < 64; r += 4)
            if (c0 + r < C && m0 + lane < M) out[(c0 + r) * out_ld + m0 + lane] = t[r][lane];
        __syncthreads();
    }
}

constexpr int64_t kMaxCols = (int64_t)1 << 31;

// strips of rows whose partials a column's scale is taken from
int64_t cols_strips(int64_t M, int64_t C)
{
    const int64_t tiles = ceil_div64(C, 64);
    int64_t n = ceil_div64(2048, tiles > 0 ? tiles : 1);
    const int64_t most = ceil_div64(M, 64);
    n = n < most ? n : most;
    return n > 0 ? (n < 256 ? n : 256) : 1;
}

template <typename T>
int launch_rows(const RqRowArgs& a, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax);
    hipLaunchKernelGGL(k_quantize_rows<T>, dim3(grid), dim3(256), 0, s, a);
    return launch_ok();
}

template <typename T>
int launch_cols(const RqRowArgs& a, hipStream_t s)
{
    const unsigned ct = (unsigned)ceil_div64(a.C, 64);
    const int64_t strips = cols_strips(a.M, a.C);
    const int64_t strip = ceil_div64(a.M, strips);
    hipLaunchKernelGGL(k_cols_stats<T>, dim3(ct, (unsigned)strips), dim3(256), 0, s, a, strip);
    hipLaunchKernelGGL(k_cols_scale, dim3((unsigned)ceil_div64(a.C, 256)), dim3(256), 0, s, a, (int)strips);
    if (a.M > 0) {
        const int64_t mt = ceil_div64(a.M, 64);
        hipLaunchKernelGGL(k_cols_codes<T>, dim3(ct, (unsigned)(mt < 1024 ? mt : 1024)), dim3(256), 0, s, a);
    }
    return launch_ok();
}

int rq_check(int32_t x_dtype, int32_t bits, int32_t mode)
{
    if (!is_float_dtype(x_dtype) || bits < 2 || bits > 8) return ISEG_ERR_ARG;
    if (mode != ISEG_SCALE_MAX && mode != ISEG_SCALE_POW2) return ISEG_ERR_ARG;
    return ISEG_OK;
}

}  // namespace

extern "C" int iseg_quantize_rows(const void* x, int32_t x_dtype, int64_t M, int64_t C, int64_t x_ld,
                                  const float* mul, int32_t bits, int32_t scale_mode, int8_t* codes,
                                  int64_t codes_ld, float* scale, int32_t* dev_status, hipStream_t stream)
{
    const int rc = rq_check(x_dtype, bits, scale_mode);
    if (rc != ISEG_OK) return rc;
    if (M < 0 || C < 0 || C >= kMaxCols || x_ld < C || codes_ld < C) return ISEG_ERR_SHAPE;
    if (M == 0) return ISEG_OK;
    if (!scale || (C > 0 && (!x || !codes))) return ISEG_ERR_ARG;
    RqRowArgs a = {};
    a.x = x; a.mul = mul; a.codes = codes; a.scale = scale;
    a.M = M; a.C = C; a.x_ld = x_ld; a.codes_ld = codes_ld; a.bits = bits; a.mode = scale_mode; a.status = dev_status;
    return x_dtype == ISEG_F32 ? launch_rows<float>(a, stream)
                               : x_dtype == ISEG_F16 ? launch_rows<f16_t>(a, stream) : launch_rows<bf16_t>(a, stream);
}

extern "C" size_t iseg_quantize_cols_ws(int64_t M, int64_t C)
{
    if (M < 0 || C < 0 || C >= kMaxCols) return 0;
    const size_t b = (size_t)cols_strips(M, C) * (size_t)C * 12;
    return b > 256 ? align256(b) : 256;
}

extern "C" int iseg_quantize_cols(const void* x, int32_t x_dtype, int64_t M, int64_t C, int64_t x_ld,
                                  const float* mul, int32_t bits, int32_t scale_mode, int8_t* codes,
                                  int64_t codes_ld, float* scale, float* sums, void* ws, size_t ws_bytes,
                                  int32_t* dev_status, hipStream_t stream)
{
    const int rc = rq_check(x_dtype, bits, scale_mode);
    if (rc != ISEG_OK) return rc;
    if (M < 0 || C < 0 || C >= kMaxCols || x_ld < C || codes_ld < M) return ISEG_ERR_SHAPE;
    if (C == 0) return ISEG_OK;
    if (!scale || (M > 0 && (!x || !codes))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_quantize_cols_ws(M, C)) return ISEG_ERR_WORKSPACE;
    RqRowArgs a = {};
    a.x = x; a.mul = mul; a.codes = codes; a.scale = scale; a.sums = sums;
    a.pmax = (uint64_t*)ws;
    a.psum = (float*)(a.pmax + cols_strips(M, C) * C);
    a.M = M; a.C = C; a.x_ld = x_ld; a.codes_ld = codes_ld; a.bits = bits; a.mode = scale_mode; a.status = dev_status;
    return x_dtype == ISEG_F32 ? launch_cols<float>(a, stream)
                               : x_dtype == ISEG_F16 ? launch_cols<f16_t>(a, stream) : launch_cols<bf16_t>(a, stream);
}

extern "C" int iseg_transpose_i8(const int8_t* in, int64_t M, int64_t C, int64_t in_ld, int8_t* out, int64_t out_ld,
                                 hipStream_t stream)
{
    if (M < 0 || C < 0 || C >= kMaxCols || in_ld < C || out_ld < M) return ISEG_ERR_SHAPE;
    if (M == 0 || C == 0) return ISEG_OK;
    if (!in || !out) return ISEG_ERR_ARG;
    const int64_t mt = ceil_div64(M, 64);
    hipLaunchKernelGGL(k_transpose_i8, dim3((unsigned)ceil_div64(C, 64), (unsigned)(mt < 1024 ? mt : 1024)),
                       dim3(256), 0, stream, in, M, C, in_ld, out, out_ld);
    return launch_ok();
}
