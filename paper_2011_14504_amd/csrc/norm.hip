// norm.hip -- layer normalization of rows, forward and backward.
//
// Both directions are bound by memory: the forward reads x once and writes y,
// the backward reads x and dy once and writes dx.  A row is held in registers
// between the statistics and the output; the mean is taken first and the
// squares around it second (a sum of squares of raw values would cancel for
// rows with an offset).
#include "rowops.h"

namespace {

struct LnArgs {
    const void *x, *gamma, *beta, *dy;
    void *y, *dx, *dgamma, *dbeta;
    float *mean, *rstd;
    float* part;                 // backward: [grid][2][C] column sums
    int64_t M, C, x_ld, y_ld, dx_ld;
    float eps;
    int32_t* status;
};

// ---------------------------------------------------------------------------
// forward: NW waves per row, VPT vectors of a row per thread
// ---------------------------------------------------------------------------
template <typename T, typename P, int NW, int VPT>
__global__ __launch_bounds__(NW * 64) void k_layernorm_fwd(LnArgs a)
{
    constexpr int N = RowVec<T>::N;
    constexpr int NT = NW * 64;
    __shared__ float red[4 * NW];
    const int tid = threadIdx.x;
    const int64_t C = a.C;
    const float inv_c = 1.f / (float)C;
    const P* gamma = (const P*)a.gamma;
    const P* beta = (const P*)a.beta;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        RowVec<T> xv[VPT];
        float s = 0.f, z = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const int64_t c = ((int64_t)j * NT + tid) * N;
            if (c + N <= C) xv[j] = row_load(x + c);
            else xv[j] = row_load_part(x + c, c < C ? (int)(C - c) : 0, (T)0.f);
        }
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) s += (float)xv[j].v[i];
        block_sum2_f32<NW>(s, z, red);
        float mean = s * inv_c;
        // squares around the mean, and the sum of the differences, whose mean
        // is what the first sum's rounding left out
        float d1 = 0.f, d2 = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int64_t c = ((int64_t)j * NT + tid) * N + i;
                const float d = c < C ? (float)xv[j].v[i] - mean : 0.f;
                d1 += d;
                d2 = fmaf(d, d, d2);
            }
        block_sum2_f32<NW>(d1, d2, red + 2 * NW);
        const float corr = d1 * inv_c;
        const float var = fmaxf(d2 * inv_c - corr * corr, 0.f);
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (tid == 0) {
            if (a.mean) a.mean[m] = mean + corr;
            if (a.rstd) a.rstd[m] = rstd;
            if (!(fabsf(d2) <= 3.4028234e38f)) set_status(a.status, ISEG_DEV_NONFINITE);
        }
        T* y = (T*)a.y + m * a.y_ld;
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const int64_t c = ((int64_t)j * NT + tid) * N;
            if (c >= C) continue;
            RowVec<T> o;
#pragma unroll
            for (int i = 0; i < N; i++) {
                const bool in = c + i < C;
                const float g = gamma && in ? (float)gamma[c + i] : 1.f;
                const float b = beta && in ? (float)beta[c + i] : 0.f;
                o.v[i] = (T)fmaf(((float)xv[j].v[i] - mean - corr) * rstd, g, b);
            }
            if (c + N <= C) row_store(y + c, o);
            else row_store_part(y + c, o, (int)(C - c));
        }
        if (NW > 1) __syncthreads();          // red is written again by the next row
    }
}

// rows longer than the registers take: three passes over the row (the second
// and third come from the caches)
template <typename T, typename P>
__global__ __launch_bounds__(1024) void k_layernorm_fwd_long(LnArgs a)
{
    __shared__ float red[64];
    const int tid = threadIdx.x;
    const int64_t C = a.C;
    const float inv_c = 1.f / (float)C;
    const P* gamma = (const P*)a.gamma;
    const P* beta = (const P*)a.beta;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        float s = 0.f, z = 0.f;
        for (int64_t c = tid; c < C; c += 1024) s += (float)x[c];
        block_sum2_f32<16>(s, z, red);
        const float mean = s * inv_c;
        float d1 = 0.f, d2 = 0.f;
        for (int64_t c = tid; c < C; c += 1024) {
            const float d = (float)x[c] - mean;
            d1 += d;
            d2 = fmaf(d, d, d2);
        }
        block_sum2_f32<16>(d1, d2, red + 32);
        const float corr = d1 * inv_c;
        const float var = fmaxf(d2 * inv_c - corr * corr, 0.f);
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (tid == 0) {
            if (a.mean) a.mean[m] = mean + corr;
            if (a.rstd) a.rstd[m] = rstd;
            if (!(fabsf(d2) <= 3.4028234e38f)) set_status(a.status, ISEG_DEV_NONFINITE);
        }
        T* y = (T*)a.y + m * a.y_ld;
        for (int64_t c = tid; c < C; c += 1024) {
            const float g = gamma ? (float)gamma[c] : 1.f;
            const float b = beta ? (float)beta[c] : 0.f;
            y[c] = (T)fmaf(((float)x[c] - mean - corr) * rstd, g, b);
        }
        __syncthreads();
    }
}

template <typename T, typename P>
int launch_fwd(const LnArgs& a, hipStream_t s)
{
    constexpr int N = RowVec<T>::N;
    const unsigned grid = (unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax);
    if (a.C <= 256 * N) hipLaunchKernelGGL((k_layernorm_fwd<T, P, 4, 1>), dim3(grid), dim3(256), 0, s, a);
    else if (a.C <= 512 * N) hipLaunchKernelGGL((k_layernorm_fwd<T, P, 4, 2>), dim3(grid), dim3(256), 0, s, a);
    else if (a.C <= 1024 * N) hipLaunchKernelGGL((k_layernorm_fwd<T, P, 4, 4>), dim3(grid), dim3(256), 0, s, a);
    else if (a.C <= 4096 * N) hipLaunchKernelGGL((k_layernorm_fwd<T, P, 16, 4>), dim3(grid), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((k_layernorm_fwd_long<T, P>), dim3(grid), dim3(1024), 0, s, a);
    return launch_ok();
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// One block walks rows b, b + grid, ... with its threads on fixed columns, so
// the column sums of dy xhat and dy stay in registers; each block leaves one
// row of partial sums that k_layernorm_param_sum adds in block order.
template <typename T, typename P, int NW, int VPT>
__global__ __launch_bounds__(NW * 64) void k_layernorm_bwd(LnArgs a)
{
    constexpr int N = RowVec<T>::N;
    constexpr int NT = NW * 64;
    __shared__ float red[4 * NW];
    const int tid = threadIdx.x;
    const int64_t C = a.C;
    const float inv_c = 1.f / (float)C;
    const P* gamma = (const P*)a.gamma;
    float dg[VPT][N], db[VPT][N];
#pragma unroll
    for (int j = 0; j < VPT; j++)
#pragma unroll
        for (int i = 0; i < N; i++) dg[j][i] = db[j][i] = 0.f;
    int flip = 0;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, flip ^= 1) {
        const T* x = (const T*)a.x + m * a.x_ld;
        const T* dy = (const T*)a.dy + m * a.y_ld;
        const float mean = a.mean[m], rstd = a.rstd[m];
        RowVec<T> xv[VPT], dv[VPT];
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const int64_t c = ((int64_t)j * NT + tid) * N;
            if (c + N <= C) {
                xv[j] = row_load(x + c);
                dv[j] = row_load(dy + c);
            } else {
                const int n = c < C ? (int)(C - c) : 0;
                xv[j] = row_load_part(x + c, n, (T)0.f);
                dv[j] = row_load_part(dy + c, n, (T)0.f);
            }
        }
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int64_t c = ((int64_t)j * NT + tid) * N + i;
                const float d = (float)dv[j].v[i];             // 0 past the row's end
                const float xh = ((float)xv[j].v[i] - mean) * rstd;
                const float g = gamma && c < C ? d * (float)gamma[c] : d;
                s1 += g;
                s2 = fmaf(g, xh, s2);
                dg[j][i] = fmaf(d, xh, dg[j][i]);
                db[j][i] += d;
            }
        block_sum2_f32<NW>(s1, s2, red + flip * 2 * NW);
        s1 *= inv_c;
        s2 *= inv_c;
        T* dx = (T*)a.dx + m * a.dx_ld;
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const int64_t c = ((int64_t)j * NT + tid) * N;
            if (c >= C) continue;
            RowVec<T> o;
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float d = (float)dv[j].v[i];
                const float xh = ((float)xv[j].v[i] - mean) * rstd;
                const float g = gamma && c + i < C ? d * (float)gamma[c + i] : d;
                o.v[i] = (T)((g - s1 - xh * s2) * rstd);
            }
            if (c + N <= C) row_store(dx + c, o);
            else row_store_part(dx + c, o, (int)(C - c));
        }
    }
    float* part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int j = 0; j < VPT; j++)
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int64_t c = ((int64_t)j * NT + tid) * N + i;
            if (c < C) {
                part[c] = dg[j][i];
                part[C + c] = db[j][i];
            }
        }
}

// rows longer than the registers take: the two row sums first ...
template <typename T, typename P>
__global__ __launch_bounds__(1024) void k_layernorm_bwd_rows(LnArgs a, float2* __restrict__ sums)
{
    __shared__ float red[32];
    const int tid = threadIdx.x;
    const P* gamma = (const P*)a.gamma;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        const T* dy = (const T*)a.dy + m * a.y_ld;
        const float mean = a.mean[m], rstd = a.rstd[m];
        float s1 = 0.f, s2 = 0.f;
        for (int64_t c = tid; c < a.C; c += 1024) {
            const float d = (float)dy[c];
            const float g = gamma ? d * (float)gamma[c] : d;
            s1 += g;
            s2 = fmaf(g, ((float)x[c] - mean) * rstd, s2);
        }
        block_sum2_f32<16>(s1, s2, red);
        if (tid == 0) sums[m] = make_float2(s1 / (float)a.C, s2 / (float)a.C);
        __syncthreads();
    }
}

// ... then dx and the column sums over tiles of 256 columns
template <typename T, typename P>
__global__ __launch_bounds__(256) void k_layernorm_bwd_cols(LnArgs a, const float2* __restrict__ sums)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.C) return;
    const P* gamma = (const P*)a.gamma;
    const float gm = gamma ? (float)gamma[c] : 1.f;
    float dg = 0.f, db = 0.f;
    for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
        const float mean = a.mean[m], rstd = a.rstd[m];
        const float2 s = sums[m];
        const float d = (float)((const T*)a.dy)[m * a.y_ld + c];
        const float xh = ((float)((const T*)a.x)[m * a.x_ld + c] - mean) * rstd;
        dg = fmaf(d, xh, dg);
        db += d;
        ((T*)a.dx)[m * a.dx_ld + c] = (T)((d * gm - s.x - xh * s.y) * rstd);
    }
    float* part = a.part + (int64_t)blockIdx.y * 2 * a.C;
    part[c] = dg;
    part[a.C + c] = db;
}

// dgamma and dbeta: the np partial rows added in order, 64 columns per block
// with the partials dealt to four waves
template <typename P>
__global__ __launch_bounds__(256) void k_layernorm_param_sum(const float* __restrict__ part, int np, int64_t C,
                                                             P* dgamma, P* dbeta)
{
    __shared__ float red[4][2][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float g = 0.f, b = 0.f;
    if (c < C)
        for (int p = w; p < np; p += 4) {
            g += part[(int64_t)p * 2 * C + c];
            b += part[(int64_t)p * 2 * C + C + c];
        }
    red[w][0][lane] = g;
    red[w][1][lane] = b;
    __syncthreads();
    if (w != 0 || c >= C) return;
    g = red[0][0][lane] + red[1][0][lane] + red[2][0][lane] + red[3][0][lane];
    b = red[0][1][lane] + red[1][1][lane] + red[2][1][lane] + red[3][1][lane];
    if (dgamma) dgamma[c] = (P)g;
    if (dbeta) dbeta[c] = (P)b;
}

int64_t ln_elem_size(int32_t t) { return t == ISEG_F32 ? 4 : 2; }

// rows that the backward holds in registers: 1024 threads with two vectors of
// x and two of dy each
bool ln_bwd_in_regs(const iseg_layernorm_geom* g) { return g->C <= 2048 * (16 / ln_elem_size(g->x_dtype)); }

// blocks that walk the rows (one row of partial column sums each)
int ln_bwd_blocks(const iseg_layernorm_geom* g)
{
    int64_t cap = ln_bwd_in_regs(g) ? 512 : 64;
    return (int)(g->M < cap ? g->M : cap);
}

template <typename T, typename P>
int launch_bwd(const LnArgs& a, const iseg_layernorm_geom* g, hipStream_t s)
{
    constexpr int N = RowVec<T>::N;
    const int nb = ln_bwd_blocks(g);
    if (nb > 0) {
        if (!ln_bwd_in_regs(g)) {
            float2* sums = (float2*)((char*)a.part + align256((size_t)nb * 2 * a.C * 4));
            const unsigned gr = (unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax);
            hipLaunchKernelGGL((k_layernorm_bwd_rows<T, P>), dim3(gr), dim3(1024), 0, s, a, sums);
            hipLaunchKernelGGL((k_layernorm_bwd_cols<T, P>), dim3((unsigned)ceil_div64(a.C, 256), nb), dim3(256), 0,
                               s, a, (const float2*)sums);
        } else if (a.C <= 256 * N) {
            hipLaunchKernelGGL((k_layernorm_bwd<T, P, 4, 1>), dim3(nb), dim3(256), 0, s, a);
        } else if (a.C <= 512 * N) {
            hipLaunchKernelGGL((k_layernorm_bwd<T, P, 4, 2>), dim3(nb), dim3(256), 0, s, a);
        } else {
            hipLaunchKernelGGL((k_layernorm_bwd<T, P, 16, 2>), dim3(nb), dim3(1024), 0, s, a);
        }
    }
    if (a.dgamma || a.dbeta)
        hipLaunchKernelGGL((k_layernorm_param_sum<P>), dim3((unsigned)ceil_div64(a.C, 64)), dim3(256), 0, s, a.part,
                           nb, a.C, (P*)a.dgamma, (P*)a.dbeta);
    return launch_ok();
}

int ln_check(const iseg_layernorm_geom* g)
{
    if (!g || !is_float_dtype(g->x_dtype) || !is_float_dtype(g->p_dtype)) return ISEG_ERR_ARG;
    if (g->M < 0 || g->C < 1 || g->C >= (int64_t)1 << 31 || g->x_ld < g->C || g->y_ld < g->C) return ISEG_ERR_SHAPE;
    return ISEG_OK;
}

}  // namespace

#define ISEG_LN_DISPATCH(fn, ...)                                                                        \
    switch (g->x_dtype * 8 + g->p_dtype) {                                                               \
    case ISEG_F32 * 8 + ISEG_F32: return fn<float, float>(__VA_ARGS__);                                  \
    case ISEG_F32 * 8 + ISEG_F16: return fn<float, f16_t>(__VA_ARGS__);                                  \
    case ISEG_F32 * 8 + ISEG_BF16: return fn<float, bf16_t>(__VA_ARGS__);                                \
    case ISEG_F16 * 8 + ISEG_F32: return fn<f16_t, float>(__VA_ARGS__);                                  \
    case ISEG_F16 * 8 + ISEG_F16: return fn<f16_t, f16_t>(__VA_ARGS__);                                  \
    case ISEG_F16 * 8 + ISEG_BF16: return fn<f16_t, bf16_t>(__VA_ARGS__);                                \
    case ISEG_BF16 * 8 + ISEG_F32: return fn<bf16_t, float>(__VA_ARGS__);                                \
    case ISEG_BF16 * 8 + ISEG_F16: return fn<bf16_t, f16_t>(__VA_ARGS__);                                \
    default: return fn<bf16_t, bf16_t>(__VA_ARGS__);                                                     \
    }

extern "C" int iseg_layernorm_fwd(const void* x, const void* gamma, const void* beta, const iseg_layernorm_geom* g,
                                  void* y, float* mean, float* rstd, int32_t* dev_status, hipStream_t stream)
{
    const int rc = ln_check(g);
    if (rc != ISEG_OK) return rc;
    if (!(g->eps > 0.f) || !(g->eps <= 3.4028234e38f)) return ISEG_ERR_ARG;
    if (g->M == 0) return ISEG_OK;
    if (!x || !y) return ISEG_ERR_ARG;
    LnArgs a = {};
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd;
    a.M = g->M; a.C = g->C; a.x_ld = g->x_ld; a.y_ld = g->y_ld; a.eps = g->eps; a.status = dev_status;
    ISEG_LN_DISPATCH(launch_fwd, a, stream)
}

extern "C" size_t iseg_layernorm_bwd_ws(const iseg_layernorm_geom* g)
{
    if (ln_check(g) != ISEG_OK) return 0;
    const size_t nb = (size_t)ln_bwd_blocks(g);
    size_t b = align256(nb * 2 * (size_t)g->C * 4);
    if (!ln_bwd_in_regs(g)) b += align256((size_t)g->M * 8);
    return b > 256 ? b : 256;
}

extern "C" int iseg_layernorm_bwd(const void* dy, const void* x, const void* gamma, const float* mean,
                                  const float* rstd, const iseg_layernorm_geom* g, void* dx, void* dgamma,
                                  void* dbeta, void* ws, size_t ws_bytes, hipStream_t stream)
{
    const int rc = ln_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->dx_ld < g->C) return ISEG_ERR_SHAPE;
    if (g->M > 0 && (!dy || !x || !mean || !rstd || !dx)) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_layernorm_bwd_ws(g)) return ISEG_ERR_WORKSPACE;
    LnArgs a = {};
    a.x = x; a.gamma = gamma; a.dy = dy; a.dx = dx; a.dgamma = dgamma; a.dbeta = dbeta;
    a.mean = (float*)mean; a.rstd = (float*)rstd; a.part = (float*)ws;
    a.M = g->M; a.C = g->C; a.x_ld = g->x_ld; a.y_ld = g->y_ld; a.dx_ld = g->dx_ld;
    ISEG_LN_DISPATCH(launch_bwd, a, g, stream)
}
