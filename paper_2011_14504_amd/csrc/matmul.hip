// matmul.hip -- int8 x int8 matrix products on MFMA with a scale for each row
// of either operand (iseg_matmul_i8).
//
// Both operands have the reduction along the row, so a 16-byte piece of a row
// is one lane's operand of v_mfma_i32_16x16x64_i8.  The int32 sums are exact,
// so any split of the reduction gives the same bits.
#include "rowops.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

struct MmArgs {
    const int8_t *a, *b;
    const float *sa, *sb, *bias;
    void* out;
    int64_t M, N, K, lda, ldb, ldc;
};

// 16 bytes of a row from column k on, zero from the row's end on
__device__ __forceinline__ v4i load16(const int8_t* row, int64_t k, int64_t K)
{
    v4i r = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&r, row + k, 16);
    } else if (k < K) {
        int8_t t[16];
#pragma unroll
        for (int i = 0; i < 16; i++) t[i] = 0;
#pragma unroll
        for (int i = 0; i < 16; i++)
            if (k + i < K) t[i] = row[k + i];
        __builtin_memcpy(&r, t, 16);
    }
    return r;
}

__device__ __forceinline__ float mm_scale(const MmArgs& p, int sum, int64_t m, int64_t n)
{
    float v = (float)sum;
    if (p.sa) v *= p.sa[m];
    if (p.sb) v *= p.sb[n];
    return p.bias ? v + p.bias[n] : v;
}

__device__ __forceinline__ int mm_swz(int row, int part) { return row * 64 + ((part ^ ((row >> 1) & 3)) << 4); }

// 64 x 64 outputs per block, 64 of the reduction per step
template <typename TO>
__global__ __launch_bounds__(256) void k_matmul_i8(MmArgs p)
{
    __shared__ __attribute__((aligned(16))) int8_t As[64 * 64], Bs[64 * 64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * 64;
    const int row = tid >> 2, part = tid & 3;
    const int lr = lane & 15, lp = lane >> 4;
    const int wm = (w >> 1) * 32, wn = (w & 1) * 32;
    const int64_t mt = ceil_div64(p.M, 64);
    for (int64_t b = blockIdx.y; b < mt; b += gridDim.y) {
        const int64_t m0 = b * 64;
        const int8_t* ar = m0 + row < p.M ? p.a + (m0 + row) * p.lda : nullptr;
        const int8_t* br = n0 + row < p.N ? p.b + (n0 + row) * p.ldb : nullptr;
        v4i acc[2][2];
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < 2; j++) acc[i][j] = (v4i){0, 0, 0, 0};
        for (int64_t k0 = 0; k0 < p.K; k0 += 64) {
            const v4i z = {0, 0, 0, 0};
            const v4i va = ar ? load16(ar, k0 + part * 16, p.K) : z;
            const v4i vb = br ? load16(br, k0 + part * 16, p.K) : z;
            __syncthreads();
            *(v4i*)&As[mm_swz(row, part)] = va;
            *(v4i*)&Bs[mm_swz(row, part)] = vb;
            __syncthreads();
            v4i fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; i++) fa[i] = *(const v4i*)&As[mm_swz(wm + i * 16 + lr, lp)];
#pragma unroll
            for (int j = 0; j < 2; j++) fb[j] = *(const v4i*)&Bs[mm_swz(wn + j * 16 + lr, lp)];
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int j = 0; j < 2; j++)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const int64_t m = m0 + wm + i * 16 + lp * 4 + r, n = n0 + wn + j * 16 + lr;
                    if (m < p.M && n < p.N) ((TO*)p.out)[m * p.ldc + n] = (TO)mm_scale(p, acc[i][j][r], m, n);
                }
    }
}

template <typename TO>
int launch_mm(const MmArgs& p, hipStream_t s)
{
    const int64_t mt = ceil_div64(p.M, 64);
    hipLaunchKernelGGL(k_matmul_i8<TO>, dim3((unsigned)ceil_div64(p.N, 64), (unsigned)(mt < 4096 ? mt : 4096)),
                       dim3(256), 0, s, p);
    return launch_ok();
}

int mm_check(const iseg_matmul_geom* g)
{
    if (!g || !is_float_dtype(g->out_dtype)) return ISEG_ERR_ARG;
    const int64_t big = (int64_t)1 << 31;
    if (g->M < 0 || g->N < 0 || g->K < 0 || g->M >= big || g->N >= big || g->lda < g->K || g->ldb < g->K ||
        g->ldc < g->N)
        return ISEG_ERR_SHAPE;
    if (g->K > 131071) return ISEG_ERR_UNSUPPORTED;
    return ISEG_OK;
}

}  // namespace

extern "C" size_t iseg_matmul_i8_ws(const iseg_matmul_geom* g)
{
    return mm_check(g) == ISEG_OK ? 256 : 0;
}

extern "C" int iseg_matmul_i8(const int8_t* a, const float* a_scale, const int8_t* b, const float* b_scale,
                              const float* bias, const iseg_matmul_geom* g, void* out, void* ws, size_t ws_bytes,
                              hipStream_t stream)
{
    const int rc = mm_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->M == 0 || g->N == 0) return ISEG_OK;
    if (!out || (g->K > 0 && (!a || !b))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_matmul_i8_ws(g)) return ISEG_ERR_WORKSPACE;
    MmArgs p = {};
    p.a = a; p.b = b; p.sa = a_scale; p.sb = b_scale; p.bias = bias; p.out = out;
    p.M = g->M; p.N = g->N; p.K = g->K; p.lda = g->lda; p.ldb = g->ldb; p.ldc = g->ldc;
    return g->out_dtype == ISEG_F32 ? launch_mm<float>(p, stream)
                                    : g->out_dtype == ISEG_F16 ? launch_mm<f16_t>(p, stream) : launch_mm<bf16_t>(p, stream);
}
