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
// forward: NW waves per row (one, or the whole block), VPT vectors of a row per
// thread.  A block walks its rows with gamma and beta in registers and the
// next row's x on its way.  16384 x 4096 bf16 49.8 us, 5.4 TB/s of x and y (a
// large copy reaches 4.8); 4 x 2048 takes 3.2 us, the latency of one load, two
// sums over a block and a store.
// ---------------------------------------------------------------------------
template <typename T, typename P, int NW, int VPT>
__global__ __launch_bounds__(NW < 4 ? 256 : NW * 64) void k_layernorm_fwd(LnArgs a)
{
    constexpr int N = RowVec<T>::N;
    constexpr int NT = NW * 64, R = NW < 4 ? 4 / NW : 1;      // threads of a row, rows of a block
    __shared__ float red[4 * NW];
    const int tid = threadIdx.x % NT;
    const int64_t C = a.C;
    const float inv_c = 1.f / (float)C;
    RowSlot<N> sl[VPT];                                       // only the last one may be short
    ParamVec<P, N> gm[VPT], bt[VPT];
#pragma unroll
    for (int j = 0; j < VPT; j++) {
        const int64_t c = ((int64_t)j * NT + tid) * N;
        sl[j] = j < VPT - 1 ? RowSlot<N>{c, 0} : row_slot<N>(c, C);
        gm[j] = param_load<P, N>((const P*)a.gamma, sl[j], 1.f);
        bt[j] = param_load<P, N>((const P*)a.beta, sl[j], 0.f);
    }
    RowVec<T> xv[VPT];
    int64_t m = (int64_t)blockIdx.x * R + threadIdx.x / NT;
    const int64_t step = (int64_t)gridDim.x * R;
    if (m < a.M) {
#pragma unroll
        for (int j = 0; j < VPT; j++) xv[j] = slot_load<T, N>((const T*)a.x + m * a.x_ld, sl[j]);
    }
    for (; m < a.M; m += step) {
        float v[VPT][N];
        float s = 0.f, z = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) v[j][i] = (float)xv[j].v[i];
        if (m + step < a.M) {
#pragma unroll
            for (int j = 0; j < VPT; j++) xv[j] = slot_load<T, N>((const T*)a.x + (m + step) * a.x_ld, sl[j]);
        }
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) s += j < VPT - 1 || i >= sl[j].dup ? v[j][i] : 0.f;
        block_sum2_f32<NW>(s, z, red);
        const float mean = s * inv_c;
        // squares around the mean, and the sum of the differences, whose mean
        // is what the first sum's rounding left out
        float d1 = 0.f, d2 = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                v[j][i] -= mean;
                const float d = j < VPT - 1 || i >= sl[j].dup ? v[j][i] : 0.f;
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
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            RowVec<T> o;
#pragma unroll
            for (int i = 0; i < N; i++)
                o.v[i] = (T)fmaf((v[j][i] - corr) * rstd, (float)gm[j].v[i], (float)bt[j].v[i]);
            if (j < VPT - 1 || sl[j].dup < N) row_store((T*)a.y + m * a.y_ld + sl[j].at, o);
        }
    }
}

// rows longer than the registers take: three passes over the row, the second
// and third from the caches (4096 x 50000 bf16 279 us, 2.9 TB/s of x and y)
template <typename T, typename P>
__global__ __launch_bounds__(1024) void k_layernorm_fwd_long(LnArgs a)
{
    constexpr int N = RowVec<T>::N, NW = 16, U = 2;
    __shared__ float red[4 * NW];
    const int64_t C = a.C;
    const float inv_c = 1.f / (float)C;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        float s = 0.f, z = 0.f;
        for (int64_t c = threadIdx.x * N; c < C; c += U * 1024 * N) {
            RowVec<T> v[U];
            RowSlot<N> sl[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                sl[u] = row_slot<N>(c + u * 1024 * N, C);
                v[u] = slot_load<T, N>(x, sl[u]);
            }
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int i = 0; i < N; i++) s += i >= sl[u].dup ? (float)v[u].v[i] : 0.f;
        }
        block_sum2_f32<NW>(s, z, red);
        const float mean = s * inv_c;
        float d1 = 0.f, d2 = 0.f;
        for (int64_t c = threadIdx.x * N; c < C; c += U * 1024 * N) {
            RowVec<T> v[U];
            RowSlot<N> sl[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                sl[u] = row_slot<N>(c + u * 1024 * N, C);
                v[u] = slot_load<T, N>(x, sl[u]);
            }
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const float d = i >= sl[u].dup ? (float)v[u].v[i] - mean : 0.f;
                    d1 += d;
                    d2 = fmaf(d, d, d2);
                }
        }
        block_sum2_f32<NW>(d1, d2, red + 2 * NW);
        const float corr = d1 * inv_c;
        const float var = fmaxf(d2 * inv_c - corr * corr, 0.f);
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[m] = mean + corr;
            if (a.rstd) a.rstd[m] = rstd;
            if (!(fabsf(d2) <= 3.4028234e38f)) set_status(a.status, ISEG_DEV_NONFINITE);
        }
        // y may be x: the last vector shares elements with another thread's, so
        // every thread stores its own only
        T* y = (T*)a.y + m * a.y_ld;
        for (int64_t c = threadIdx.x * N; c < C; c += 1024 * N) {
            const RowSlot<N> sl = row_slot<N>(c, C);
            const RowVec<T> v = row_load(x + sl.at);
            const ParamVec<P, N> gm = param_load<P, N>((const P*)a.gamma, sl, 1.f), bt = param_load<P, N>((const P*)a.beta, sl, 0.f);
            RowVec<T> o;
#pragma unroll
            for (int i = 0; i < N; i++)
                o.v[i] = (T)fmaf(((float)v.v[i] - mean - corr) * rstd, (float)gm.v[i], (float)bt.v[i]);
            if (sl.dup == 0) {
                row_store(y + sl.at, o);
            } else {
#pragma unroll
                for (int i = 0; i < N; i++)
                    if (i >= sl.dup) y[sl.at + i] = o.v[i];
            }
        }
    }
}

// rows shorter than a vector, one per thread (100000 x 3 fp32 3.5 us; with a
// wave per row 27)
template <typename T, typename P>
__global__ __launch_bounds__(256) void k_layernorm_fwd_narrow(LnArgs a)
{
    const int C = (int)a.C;
    const float inv_c = 1.f / (float)C;
    for (int64_t m = blockIdx.x * (int64_t)256 + threadIdx.x; m < a.M; m += (int64_t)gridDim.x * 256) {
        const T* x = (const T*)a.x + m * a.x_ld;
        float s = 0.f, d1 = 0.f, d2 = 0.f;
        for (int c = 0; c < C; c++) s += (float)x[c];
        const float mean = s * inv_c;
        for (int c = 0; c < C; c++) {
            const float d = (float)x[c] - mean;
            d1 += d;
            d2 = fmaf(d, d, d2);
        }
        const float corr = d1 * inv_c;
        const float var = fmaxf(d2 * inv_c - corr * corr, 0.f);
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (a.mean) a.mean[m] = mean + corr;
        if (a.rstd) a.rstd[m] = rstd;
        if (!(fabsf(d2) <= 3.4028234e38f)) set_status(a.status, ISEG_DEV_NONFINITE);
        T* y = (T*)a.y + m * a.y_ld;
        for (int c = 0; c < C; c++) {
            const float g = a.gamma ? (float)((const P*)a.gamma)[c] : 1.f;
            const float b = a.beta ? (float)((const P*)a.beta)[c] : 0.f;
            y[c] = (T)fmaf(((float)x[c] - mean - corr) * rstd, g, b);
        }
    }
}

// Waves and vectors per row, by the row's vectors.  16384 x 4096 bf16 (512
// vectors): four waves of two 48.9 us (5.5 TB/s), one wave of eight 57;
// 32768 x 2048: four of one 50.6, one of four 51.5; 32768 x 1024: one of two
// 28.9.  More blocks than the chip holds at once reload gamma and beta for
// fewer rows each: 55 us with a block per row in the first case.
template <typename T, typename P, int NW, int VPT>
int fwd_grid(const LnArgs& a, unsigned cap, hipStream_t s)
{
    constexpr int R = NW < 4 ? 4 / NW : 1;
    if (!slots_fit<T, NW, VPT>(a.C)) return ISEG_ERR_UNSUPPORTED;
    const int64_t nb = ceil_div64(a.M, R);
    hipLaunchKernelGGL((k_layernorm_fwd<T, P, NW, VPT>), dim3((unsigned)(nb < cap ? nb : cap)),
                       dim3(NW < 4 ? 256 : NW * 64), 0, s, a);
    return launch_ok();
}

template <typename T, typename P>
int launch_fwd(const LnArgs& a, hipStream_t s)
{
    constexpr int N = RowVec<T>::N;
    const int64_t v = ceil_div64(a.C, N);
    const unsigned grid = (unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax);
    if (a.C < N) {
        hipLaunchKernelGGL((k_layernorm_fwd_narrow<T, P>), dim3(grid_for(a.M, 256, 4096)), dim3(256), 0, s, a);
        return launch_ok();
    }
    if (v <= 64) return fwd_grid<T, P, 1, 1>(a, 2048, s);
    if (v <= 128) return fwd_grid<T, P, 1, 2>(a, 2048, s);
    if (v <= 256) return fwd_grid<T, P, 4, 1>(a, 4096, s);
    if (v <= 512) return fwd_grid<T, P, 4, 2>(a, 4096, s);
    if (v <= 768) return fwd_grid<T, P, 4, 3>(a, 2048, s);
    if (v <= 1024) return fwd_grid<T, P, 4, 4>(a, 2048, s);
    if (v <= 1536) return fwd_grid<T, P, 8, 3>(a, 1024, s);
    if (v <= 2048) return fwd_grid<T, P, 8, 4>(a, 1024, s);
    // gamma and beta of float32 beside vectors of eight do not fit (2048 x 16384
    // fp32 48 us, 101 in three passes; 4096 x 20000 bf16 64 and 116)
    if constexpr (N == 4 || sizeof(P) == 2) {
        if (v <= 3 * 1024) return fwd_grid<T, P, 16, 3>(a, 512, s);
        if (v <= 4096) return fwd_grid<T, P, 16, 4>(a, 512, s);
    }
    hipLaunchKernelGGL((k_layernorm_fwd_long<T, P>), dim3(grid), dim3(1024), 0, s, a);
    return launch_ok();
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// One block walks rows b, b + grid, ... with its threads on fixed columns, so
// gamma and the column sums of dy xhat and dy stay in registers and the next
// row's x and dy are on their way; each block leaves one row of partial sums
// that k_layernorm_param_sum adds in block order.  5003 x 1537 fp32 20.1 us with
// the sum, 4.6 TB/s of x, dy and dx.
template <typename T, typename P, int NW, int VPT>
__global__ __launch_bounds__(NW * 64) void k_layernorm_bwd(LnArgs a)
{
    constexpr int N = RowVec<T>::N;
    constexpr int NT = NW * 64;
    __shared__ float red[4 * NW];
    const int tid = threadIdx.x;
    const int64_t C = a.C;
    const float inv_c = 1.f / (float)C;
    RowSlot<N> sl[VPT];                                       // only the last one may be short
    ParamVec<P, N> gm[VPT];
    float dg[VPT][N], db[VPT][N];
#pragma unroll
    for (int j = 0; j < VPT; j++) {
        const int64_t c = ((int64_t)j * NT + tid) * N;
        sl[j] = j < VPT - 1 ? RowSlot<N>{c, 0} : row_slot<N>(c, C);
        gm[j] = param_load<P, N>((const P*)a.gamma, sl[j], 1.f);
#pragma unroll
        for (int i = 0; i < N; i++) dg[j][i] = db[j][i] = 0.f;
    }
    RowVec<T> xv[VPT], dv[VPT];
    float mean_n = 0.f, rstd_n = 0.f;
    auto fetch = [&](int64_t m) {
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            xv[j] = slot_load<T, N>((const T*)a.x + m * a.x_ld, sl[j]);
            dv[j] = slot_load<T, N>((const T*)a.dy + m * a.y_ld, sl[j]);
        }
        mean_n = a.mean[m];
        rstd_n = a.rstd[m];
    };
    if (blockIdx.x < a.M) fetch(blockIdx.x);
    int flip = 0;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, flip ^= 1) {
        const float mean = mean_n, rstd = rstd_n;
        float xh[VPT][N], g[VPT][N];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float d = (float)dv[j].v[i];
                xh[j][i] = ((float)xv[j].v[i] - mean) * rstd;
                g[j][i] = d * (float)gm[j].v[i];
                const bool own = j < VPT - 1 || i >= sl[j].dup;
                const float go = own ? g[j][i] : 0.f, dn = own ? d : 0.f;
                s1 += go;
                s2 = fmaf(go, xh[j][i], s2);
                dg[j][i] = fmaf(dn, xh[j][i], dg[j][i]);
                db[j][i] += dn;
            }
        if (m + gridDim.x < a.M) fetch(m + gridDim.x);
        block_sum2_f32<NW>(s1, s2, red + flip * 2 * NW);
        s1 *= inv_c;
        s2 *= inv_c;
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            RowVec<T> o;
#pragma unroll
            for (int i = 0; i < N; i++) o.v[i] = (T)((g[j][i] - s1 - xh[j][i] * s2) * rstd);
            if (j < VPT - 1 || sl[j].dup < N) row_store((T*)a.dx + m * a.dx_ld + sl[j].at, o);
        }
    }
    if (gridDim.x == 1) {                                     // a few rows: the block's sums are the sums
#pragma unroll
        for (int j = 0; j < VPT; j++)
#pragma unroll
            for (int i = 0; i < N; i++)
                if (i >= sl[j].dup) {
                    if (a.dgamma) ((P*)a.dgamma)[sl[j].at + i] = (P)dg[j][i];
                    if (a.dbeta) ((P*)a.dbeta)[sl[j].at + i] = (P)db[j][i];
                }
        return;
    }
    float* part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int j = 0; j < VPT; j++) {
        if (sl[j].dup == 0) {
            __builtin_memcpy(part + sl[j].at, dg[j], sizeof(dg[j]));
            __builtin_memcpy(part + C + sl[j].at, db[j], sizeof(db[j]));
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                if (i >= sl[j].dup) {
                    part[sl[j].at + i] = dg[j][i];
                    part[C + sl[j].at + i] = db[j][i];
                }
        }
    }
}

// rows longer than the registers take: the two row sums first ...
template <typename T, typename P>
__global__ __launch_bounds__(1024) void k_layernorm_bwd_rows(LnArgs a, float2* __restrict__ sums)
{
    constexpr int N = RowVec<T>::N;
    __shared__ float red[32];
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        const T* dy = (const T*)a.dy + m * a.y_ld;
        const float mean = a.mean[m], rstd = a.rstd[m];
        float s1 = 0.f, s2 = 0.f;
        for (int64_t c = threadIdx.x * N; c < a.C; c += 1024 * N) {
            const RowSlot<N> sl = row_slot<N>(c, a.C);
            const RowVec<T> xv = row_load(x + sl.at), dv = row_load(dy + sl.at);
            const ParamVec<P, N> gm = param_load<P, N>((const P*)a.gamma, sl, 1.f);
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float g = i >= sl.dup ? (float)dv.v[i] * (float)gm.v[i] : 0.f;
                s1 += g;
                s2 = fmaf(g, ((float)xv.v[i] - mean) * rstd, s2);
            }
        }
        block_sum2_f32<16>(s1, s2, red);
        if (threadIdx.x == 0) sums[m] = make_float2(s1 / (float)a.C, s2 / (float)a.C);
        __syncthreads();
    }
}

// ... then dx and the column sums: a wave takes 64 vectors of columns, its rows
// one after the other.  Both kernels read x and dy: 4096 x 32768 bf16 276 us,
// 4.9 TB/s of what they move
template <typename T, typename P>
__global__ __launch_bounds__(64) void k_layernorm_bwd_cols(LnArgs a, const float2* __restrict__ sums)
{
    constexpr int N = RowVec<T>::N;
    const RowSlot<N> sl = row_slot<N>(((int64_t)blockIdx.x * 64 + threadIdx.x) * N, a.C);
    if (sl.dup == N) return;
    const ParamVec<P, N> gm = param_load<P, N>((const P*)a.gamma, sl, 1.f);
    float dg[N], db[N];
#pragma unroll
    for (int i = 0; i < N; i++) dg[i] = db[i] = 0.f;
    RowVec<T> xn = row_load((const T*)a.x + blockIdx.y * a.x_ld + sl.at), dn = row_load((const T*)a.dy + blockIdx.y * a.y_ld + sl.at);
    for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
        const RowVec<T> xv = xn, dv = dn;
        if (m + gridDim.y < a.M) {
            xn = row_load((const T*)a.x + (m + gridDim.y) * a.x_ld + sl.at);
            dn = row_load((const T*)a.dy + (m + gridDim.y) * a.y_ld + sl.at);
        }
        const float mean = a.mean[m], rstd = a.rstd[m];
        const float2 s = sums[m];
        RowVec<T> o;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float d = (float)dv.v[i], xh = ((float)xv.v[i] - mean) * rstd;
            dg[i] = fmaf(d, xh, dg[i]);
            db[i] += d;
            o.v[i] = (T)((d * (float)gm.v[i] - s.x - xh * s.y) * rstd);
        }
        T* dx = (T*)a.dx + m * a.dx_ld + sl.at;
        // dx may be dy or x: of a vector that shares elements with another
        // thread's, each stores its own only
        if (sl.dup == 0) {
            row_store(dx, o);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                if (i >= sl.dup) dx[i] = o.v[i];
        }
    }
    float* part = a.part + (int64_t)blockIdx.y * 2 * a.C + sl.at;
#pragma unroll
    for (int i = 0; i < N; i++)
        if (i >= sl.dup) {
            part[i] = dg[i];
            part[a.C + i] = db[i];
        }
}

// rows shorter than a vector, one per thread
template <typename T, typename P>
__global__ __launch_bounds__(256) void k_layernorm_bwd_narrow(LnArgs a)
{
    constexpr int N = RowVec<T>::N;
    __shared__ float red[2][8];
    const int C = (int)a.C;
    const float inv_c = 1.f / (float)C;
    float gm[N], dg[N], db[N];
#pragma unroll
    for (int i = 0; i < N; i++) {
        gm[i] = a.gamma && i < C ? (float)((const P*)a.gamma)[i] : 1.f;
        dg[i] = db[i] = 0.f;
    }
    for (int64_t m = blockIdx.x * (int64_t)256 + threadIdx.x; m < a.M; m += (int64_t)gridDim.x * 256) {
        const float mean = a.mean[m], rstd = a.rstd[m];
        float g[N], xh[N], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float d = i < C ? (float)((const T*)a.dy)[m * a.y_ld + i] : 0.f;
            xh[i] = i < C ? ((float)((const T*)a.x)[m * a.x_ld + i] - mean) * rstd : 0.f;
            g[i] = d * gm[i];
            s1 += g[i];
            s2 = fmaf(g[i], xh[i], s2);
            dg[i] = fmaf(d, xh[i], dg[i]);
            db[i] += d;
        }
        s1 *= inv_c;
        s2 *= inv_c;
#pragma unroll
        for (int i = 0; i < N; i++)
            if (i < C) ((T*)a.dx)[m * a.dx_ld + i] = (T)((g[i] - s1 - xh[i] * s2) * rstd);
    }
    float* part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int i = 0; i < N; i++) {
        block_sum2_f32<4>(dg[i], db[i], red[i & 1]);
        if (i < C && threadIdx.x == 0) {
            part[i] = dg[i];
            part[C + i] = db[i];
        }
    }
}

// dgamma (blockIdx.y = 0) or dbeta (1): the np partial rows added in one
// order, 64 columns per block, the rows dealt to its sixteen waves
template <typename P>
__global__ __launch_bounds__(1024) void k_layernorm_param_sum(const float* __restrict__ part, int np, int64_t C,
                                                              P* dgamma, P* dbeta)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    P* out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const float* col = part + blockIdx.y * C + (c < C ? c : C - 1);
    float s = 0.f;
    for (int p0 = w; p0 < np; p0 += 16 * 8) {
        float t[8];
#pragma unroll
        for (int u = 0; u < 8; u++) t[u] = col[(int64_t)(p0 + 16 * u < np ? p0 + 16 * u : p0) * 2 * C];
#pragma unroll
        for (int u = 0; u < 8; u++) s += p0 + 16 * u < np ? t[u] : 0.f;
    }
    red[w][lane] = s;
    __syncthreads();
    if (w != 0 || c >= C) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) s += red[i][lane];
    out[c] = (P)s;
}

// rows that the backward holds in registers: three vectors of float32 for each
// thread of 16 waves, 2048 of a shorter type, whose vectors take twice the registers.  4096
// x 16384 bf16 95 us (4.2 TB/s); 4096 x 20000, in two passes, 187 (2.6)
int64_t ln_vectors(const iseg_layernorm_geom* g) { return ceil_div64(g->C, g->x_dtype == ISEG_F32 ? 4 : 8); }

bool ln_bwd_in_regs(const iseg_layernorm_geom* g)
{
    return g->x_dtype == ISEG_F32 ? g->C >= 4 && ln_vectors(g) <= 3 * 1024 : g->C >= 8 && ln_vectors(g) <= 2048;
}

// Blocks that walk the rows, each of which leaves 2 C floats of partial sums:
// one per CU where a block's rows fill it, more where they are short.  bf16,
// with the sum over the partials: 8192 x 4096 46.5 us with 256 blocks of 8
// waves, 50.5 with 512; 1024 x 2048 (fp32) 12.5 and 15.7; 16384 x 2048 of 4
// waves 61.6 / 47.0 / 49.0 with 256 / 512 / 768; 32768 x 512 of one wave 38.7
// / 35.8 / 42.7 with 1024 / 1536 / twice that.
int ln_bwd_blocks(const iseg_layernorm_geom* g)
{
    const int64_t v = ln_vectors(g);
    // few and short: one block (25 GB/s), and no second kernel (5 us)
    if (ln_bwd_in_regs(g) && g->M <= 8 && g->M * v <= 4096) return g->M > 0;
    const int64_t cap = !ln_bwd_in_regs(g) ? 64 : v <= 64 ? 1536 : v <= 128 ? 1024 : v <= 256 ? 512 : 256;
    return (int)(g->M < cap ? g->M : cap);
}

template <typename T, typename P, int NW, int VPT>
int bwd_grid(const LnArgs& a, int nb, hipStream_t s)
{
    if (!slots_fit<T, NW, VPT>(a.C)) return ISEG_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((k_layernorm_bwd<T, P, NW, VPT>), dim3(nb), dim3(NW * 64), 0, s, a);
    return launch_ok();
}

template <typename T, typename P>
int launch_bwd(const LnArgs& a, const iseg_layernorm_geom* g, hipStream_t s)
{
    constexpr int N = RowVec<T>::N;
    const int nb = ln_bwd_blocks(g);
    const int64_t v = ceil_div64(a.C, N);
    if (nb > 0) {
        int rc;
        if (a.C < N) {
            hipLaunchKernelGGL((k_layernorm_bwd_narrow<T, P>), dim3(nb), dim3(256), 0, s, a);
            rc = launch_ok();
        } else if (!ln_bwd_in_regs(g)) {
            float2* sums = (float2*)((char*)a.part + align256((size_t)nb * 2 * a.C * 4));
            const unsigned gr = (unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax);
            hipLaunchKernelGGL((k_layernorm_bwd_rows<T, P>), dim3(gr), dim3(1024), 0, s, a, sums);
            hipLaunchKernelGGL((k_layernorm_bwd_cols<T, P>), dim3((unsigned)ceil_div64(a.C, 64 * N), nb), dim3(64), 0,
                               s, a, (const float2*)sums);
            rc = launch_ok();
        } else if (v <= 64) {
            rc = bwd_grid<T, P, 1, 1>(a, nb, s);
        } else if (v <= 128) {
            rc = bwd_grid<T, P, 1, 2>(a, nb, s);
        } else if (v <= 256) {
            rc = bwd_grid<T, P, 4, 1>(a, nb, s);
        } else if (v <= 512) {
            rc = bwd_grid<T, P, 8, 1>(a, nb, s);
        } else if (v <= 1024) {
            rc = bwd_grid<T, P, 8, 2>(a, nb, s);
        } else if (v <= 1536) {
            rc = bwd_grid<T, P, 8, 3>(a, nb, s);
        } else if (v <= 2048) {
            rc = bwd_grid<T, P, 8, 4>(a, nb, s);
        } else if constexpr (N == 4) {
            rc = bwd_grid<T, P, 16, 3>(a, nb, s);
        } else {
            rc = ISEG_ERR_UNSUPPORTED;                        // ln_bwd_in_regs has none
        }
        if (rc != ISEG_OK) return rc;
    }
    if ((a.dgamma || a.dbeta) && !(nb == 1 && ln_bwd_in_regs(g)))
        hipLaunchKernelGGL((k_layernorm_param_sum<P>), dim3((unsigned)ceil_div64(a.C, 64), 2), dim3(1024), 0, s, a.part,
                           nb, a.C, (P*)a.dgamma, (P*)a.dbeta);
    return launch_ok();
}

int ln_check(const iseg_layernorm_geom* g)
{
    if (!g || !is_float_dtype(g->x_dtype) || !is_float_dtype(g->p_dtype)) return ISEG_ERR_ARG;
    if (g->M < 0 || g->C < 1 || g->C >= (int64_t)1 << 31 || g->x_ld < g->C || g->y_ld < g->C) return ISEG_ERR_SHAPE;
    if (g->reserved) return ISEG_ERR_ARG;
    return g->C <= (int64_t)1 << 27 ? ISEG_OK : ISEG_ERR_UNSUPPORTED;      // a launch's threads
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
    else if (nb <= 1) return kNoWs;
    return ws_used(b);
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
