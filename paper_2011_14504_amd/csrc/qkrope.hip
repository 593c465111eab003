// qkrope.hip -- norms of queries and keys for each head, with the rotation of
// their positions in the same pass, and the backward (iseg_qk_norm_rope_fwd,
// iseg_qk_norm_rope_bwd).
//
// A head's row is dealt to a group of lanes in slots of two vectors that belong
// together: (i, i + R / 2) of a rotated half, two neighbours otherwise.  So a
// rotation never leaves its lane, and a row is read and written once.
#include "rowops.h"

namespace {

constexpr int kTableMax = 2048;      // sines and cosines of a block (16 KB of LDS)
constexpr int kBwdBlocks = 1024;     // of the backward, each with partial sums of gamma's gradient

struct QrSide {                      // one of q and k
    const void *x, *dy, *gamma;
    void* out;                       // y, or dx
    float* part;                     // backward: [blocks][D] partial sums of gamma's gradient
    void* dgamma;
    int64_t H, x_ld, x_hs, dy_ld, dy_hs, o_ld, o_hs;
    int32_t tokens;                  // of a block's turn
    int32_t blocks;
};

struct QrArgs {
    QrSide side[2];
    const void* pos;
    const float* freq;
    int64_t T;
    int32_t D, R, pairs, norm, pos64;
    float eps, mscale;
    int32_t* status;
};

// sine and cosine of pos * freq: the angle is formed in turns and reduced in 64
// bits (at 2^31 radians the fraction of a turn is still good to 2^-24), and what its
// float32 leaves off, up to 2^-25 half-turns, is turned by afterwards
__device__ __forceinline__ float2 turn_of(int64_t pos, float freq, float mscale)
{
    double t = (double)pos * (double)freq * 0.15915494309189533577;
    t = 2.0 * (t - rint(t));
    const float hi = (float)t, lo = (float)(t - (double)hi) * 3.14159265f;
    float s, c;
    sincospif(hi, &s, &c);
    return {fmaf(-s, lo, c) * mscale, fmaf(c, lo, s) * mscale};
}

template <typename T, int N>
struct SlotVec {
    T v[N];
};

template <typename T, int N>
__device__ __forceinline__ void slot_get(const T* p, float* f)
{
    SlotVec<T, N> r;
    __builtin_memcpy(&r, p, sizeof(r));
#pragma unroll
    for (int i = 0; i < N; i++) f[i] = (float)r.v[i];
}

template <typename T, int N>
__device__ __forceinline__ void slot_put(T* p, const float* f)
{
    SlotVec<T, N> r;
#pragma unroll
    for (int i = 0; i < N; i++) r.v[i] = (T)f[i];
    __builtin_memcpy(p, &r, sizeof(r));
}

// where a slot's two vectors lie in the row; -1: none
struct SlotAt {
    int a, b;
    bool turned;
};

template <int N>
__device__ __forceinline__ SlotAt slot_at(int slot, int D, int R, bool pairs)
{
    SlotAt s;
    const int halves = pairs ? 0 : R / (2 * N);
    if (slot < halves) {
        s = {slot * N, R / 2 + slot * N, true};
    } else {
        const int at = (pairs ? 0 : R) + (slot - halves) * 2 * N;
        s = {at < D ? at : -1, at + N < D ? at + N : -1, false};
    }
    return s;
}

// Rotates a slot (or back) by the block's table of the token.  pairs: each
// vector by itself, those inside the first R elements.
template <int N>
__device__ __forceinline__ void slot_turn(float* a, float* b, const SlotAt& s, const float2* tab, int R, bool pairs,
                                          bool back)
{
    const float sg = back ? -1.f : 1.f;
    if (s.turned) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float2 t = tab[s.a + i];
            const float u = a[i], v = b[i], sn = sg * t.y;
            a[i] = u * t.x - v * sn;
            b[i] = u * sn + v * t.x;
        }
    } else if (pairs) {
        if constexpr (N == 1) {
            if (s.a >= 0 && s.a < R) {
                const float2 t = tab[s.a >> 1];
                const float u = *a, v = *b, sn = sg * t.y;
                *a = u * t.x - v * sn;
                *b = u * sn + v * t.x;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float* p = h ? b : a;
                const int at = h ? s.b : s.a;
                if (at >= 0 && at < R) {
#pragma unroll
                    for (int i = 0; i < N; i += 2) {
                        const float2 t = tab[(at + i) >> 1];
                        const float u = p[i], v = p[i + 1], sn = sg * t.y;
                        p[i] = u * t.x - v * sn;
                        p[i + 1] = u * sn + v * t.x;
                    }
                }
            }
        }
    }
}

// sum over the LPR neighbouring lanes of a row, the same in each
template <int LPR>
__device__ __forceinline__ float row_sum(float v)
{
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// N elements a vector, LPR lanes a row, SPL slots a lane.  blockIdx.y: q or k.
// A block takes `tokens` tokens with all their heads at a time, whose sines and
// cosines it forms once.
//
// Bound by memory: 16001 tokens of 40 heads of 128 bf16, 328 MB, in 69 to 73 us, 4.5 to
// 4.7 TB/s; the backward of 8192 tokens of 32 heads of 96 float32, 302 MB, in 61 us,
// 4.9 TB/s.  8 tokens: 4.7 us, a chain of loads, sines and two barriers.
template <typename T, typename P, int N, int LPR, int SPL, bool BWD>
__global__ __launch_bounds__(256) void k_qk_norm_rope(QrArgs a)
{
    __shared__ float2 tab[kTableMax];
    const QrSide& sd = a.side[blockIdx.y];
    if ((int)blockIdx.x >= sd.blocks) return;
    constexpr int RPB = 256 / LPR;
    const int lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
    const int half = a.R / 2, H = (int)sd.H;
    SlotAt at[SPL];
    float ga[SPL][N], gb[SPL][N];                  // gamma
    float da[SPL][N], db[SPL][N];                  // BWD: gamma's gradient
#pragma unroll
    for (int j = 0; j < SPL; j++) {
        at[j] = slot_at<N>(lane + j * LPR, a.D, a.R, a.pairs);
#pragma unroll
        for (int i = 0; i < N; i++) {
            ga[j][i] = gb[j][i] = 1.f;
            da[j][i] = db[j][i] = 0.f;
        }
        if (sd.gamma) {
            if (at[j].a >= 0) slot_get<P, N>((const P*)sd.gamma + at[j].a, ga[j]);
            if (at[j].b >= 0) slot_get<P, N>((const P*)sd.gamma + at[j].b, gb[j]);
        }
    }
    SlotVec<T, N> na[SPL], nb[SPL];
#pragma unroll
    for (int j = 0; j < SPL; j++)
#pragma unroll
        for (int i = 0; i < N; i++) na[j].v[i] = nb[j].v[i] = (T)0.f;
    const int64_t groups = ceil_div64(a.T, sd.tokens);
    for (int64_t grp = blockIdx.x; grp < groups; grp += sd.blocks) {
        const int64_t t0 = grp * sd.tokens;
        const int nt = (int)(a.T - t0 < sd.tokens ? a.T - t0 : sd.tokens);
        // forward: a row ahead of the one that is turned (16001 x 40 heads of 128 bf16 71
        // us, without 80; the backward, with two rows of each, is slower with it: 65, 60)
        auto fetch = [&](int r) {
            if (BWD && !a.norm) return;
            const int t = r / H, h = r - t * H;
            const T* x = (const T*)sd.x + (t0 + t) * sd.x_ld + h * sd.x_hs;
#pragma unroll
            for (int j = 0; j < SPL; j++) {
                if (at[j].a >= 0) __builtin_memcpy(&na[j], x + at[j].a, sizeof(na[j]));
                if (at[j].b >= 0) __builtin_memcpy(&nb[j], x + at[j].b, sizeof(nb[j]));
            }
        };
        if (!BWD && sub < nt * H) fetch(sub);
        __syncthreads();                           // the table's last readers are done
        for (int i = threadIdx.x; i < nt * half; i += 256) {
            const int t = i / half;
            const int64_t p = a.pos64 ? ((const int64_t*)a.pos)[t0 + t] : ((const int32_t*)a.pos)[t0 + t];
            tab[i] = turn_of(p, a.freq[i - t * half], a.mscale);
        }
        __syncthreads();
        for (int r = sub; r < nt * H; r += RPB) {
            const int t = r / H, h = r - t * H;
            T* out = (T*)sd.out + (t0 + t) * sd.o_ld + h * sd.o_hs;
            const float2* tb = tab + t * half;
            float xa[SPL][N], xb[SPL][N];
            float ss = 0.f;
            if (BWD) fetch(r);
#pragma unroll
            for (int j = 0; j < SPL; j++)
#pragma unroll
                for (int i = 0; i < N; i++) {
                    xa[j][i] = (float)na[j].v[i];
                    xb[j][i] = (float)nb[j].v[i];
                }
            if (!BWD && r + RPB < nt * H) fetch(r + RPB);
            if constexpr (!BWD) {
                if (a.norm) {
#pragma unroll
                    for (int j = 0; j < SPL; j++)
#pragma unroll
                        for (int i = 0; i < N; i++) ss += xa[j][i] * xa[j][i] + xb[j][i] * xb[j][i];
                    ss = row_sum<LPR>(ss);
                    const float mean = ss / (float)a.D + a.eps;
                    if (!(mean >= 1.17549435e-38f && ss <= 3.4028234e38f) && lane == 0) set_status(a.status, ISEG_DEV_NONFINITE);
                    const float rs = 1.f / sqrtf(mean);
#pragma unroll
                    for (int j = 0; j < SPL; j++)
#pragma unroll
                        for (int i = 0; i < N; i++) {
                            xa[j][i] *= rs * ga[j][i];
                            xb[j][i] *= rs * gb[j][i];
                        }
                }
#pragma unroll
                for (int j = 0; j < SPL; j++) {
                    slot_turn<N>(xa[j], xb[j], at[j], tb, a.R, a.pairs, false);
                    if (at[j].a >= 0) slot_put<T, N>(out + at[j].a, xa[j]);
                    if (at[j].b >= 0) slot_put<T, N>(out + at[j].b, xb[j]);
                }
            } else {
                const T* dy = (const T*)sd.dy + (t0 + t) * sd.dy_ld + h * sd.dy_hs;
                float ya[SPL][N], yb[SPL][N];
                float dot = 0.f;
#pragma unroll
                for (int j = 0; j < SPL; j++) {
#pragma unroll
                    for (int i = 0; i < N; i++) ya[j][i] = yb[j][i] = 0.f;
                    if (at[j].a >= 0) slot_get<T, N>(dy + at[j].a, ya[j]);
                    if (at[j].b >= 0) slot_get<T, N>(dy + at[j].b, yb[j]);
                    slot_turn<N>(ya[j], yb[j], at[j], tb, a.R, a.pairs, true);
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        ss += xa[j][i] * xa[j][i] + xb[j][i] * xb[j][i];
                        dot += ya[j][i] * ga[j][i] * xa[j][i] + yb[j][i] * gb[j][i] * xb[j][i];
                    }
                }
                if (a.norm) {
                    ss = row_sum<LPR>(ss);
                    dot = row_sum<LPR>(dot);
                    const float rs = 1.f / sqrtf(ss / (float)a.D + a.eps);
                    const float k = dot / (float)a.D * rs * rs;
#pragma unroll
                    for (int j = 0; j < SPL; j++)
#pragma unroll
                        for (int i = 0; i < N; i++) {
                            da[j][i] += ya[j][i] * (xa[j][i] * rs);
                            db[j][i] += yb[j][i] * (xb[j][i] * rs);
                            ya[j][i] = rs * (ya[j][i] * ga[j][i] - xa[j][i] * k);
                            yb[j][i] = rs * (yb[j][i] * gb[j][i] - xb[j][i] * k);
                        }
                }
#pragma unroll
                for (int j = 0; j < SPL; j++) {
                    if (at[j].a >= 0) slot_put<T, N>(out + at[j].a, ya[j]);
                    if (at[j].b >= 0) slot_put<T, N>(out + at[j].b, yb[j]);
                }
            }
        }
    }
    if constexpr (BWD) {
        if (!sd.part) return;
        // the block's rows one after the other in a fixed order: over a wave's
        // groups of lanes by exchange, over its waves through LDS
        __shared__ float red[4][LPR * SPL * 2 * N];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int j = 0; j < SPL; j++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                float u = da[j][i], v = db[j][i];
#pragma unroll
                for (int o = LPR; o < 64; o <<= 1) {
                    u += __shfl_xor(u, o, 64);
                    v += __shfl_xor(v, o, 64);
                }
                if ((threadIdx.x & 63) < LPR) {
                    red[wave][((lane + j * LPR) * 2) * N + i] = u;
                    red[wave][((lane + j * LPR) * 2 + 1) * N + i] = v;
                }
            }
        __syncthreads();
        for (int e = threadIdx.x; e < LPR * SPL * 2 * N; e += 256) {
            const SlotAt s = slot_at<N>(e / (2 * N), a.D, a.R, a.pairs);
            const int d = (e / N) & 1 ? s.b : s.a;
            if (d >= 0) sd.part[(int64_t)blockIdx.x * a.D + d + e % N] = red[0][e] + red[1][e] + red[2][e] + red[3][e];
        }
    }
}

// gamma's gradient: the blocks' partial sums, 64 runs of them side by side, each by
// halves and then the runs by eights in float64 (one after the other in float32 they
// were the larger part of the gradient's error).  5.5 us; one thread a column 33.
// blockIdx.y: q or k.
template <typename P>
__global__ __launch_bounds__(1024) void k_qk_dgamma(QrArgs a)
{
    __shared__ double red[64][16];
    const QrSide& sd = a.side[blockIdx.y];
    if (!sd.dgamma) return;
    const int c = threadIdx.x & 15, seg = threadIdx.x >> 4, d = blockIdx.x * 16 + c;
    const int per = (sd.blocks + 63) / 64, b0 = seg * per;
    double s = 0.0;
    if (d < a.D) {
        float v[kBwdBlocks / 64];
#pragma unroll
        for (int i = 0; i < kBwdBlocks / 64; i++) v[i] = i < per && b0 + i < sd.blocks ? sd.part[(int64_t)(b0 + i) * a.D + d] : 0.f;
#pragma unroll
        for (int n = kBwdBlocks / 128; n > 0; n /= 2)
#pragma unroll
            for (int i = 0; i < n; i++) v[i] += v[i + n];
        s = v[0];
    }
    red[seg][c] = s;
    __syncthreads();
    // eight runs by eight threads, then theirs
    s = 0.0;
    if (seg < 8)
#pragma unroll
        for (int i = 0; i < 8; i++) s += red[seg * 8 + i][c];
    __syncthreads();
    if (seg < 8) red[seg][c] = s;
    __syncthreads();
    if (seg == 0 && d < a.D) {
#pragma unroll
        for (int i = 1; i < 8; i++) s += red[i][c];
        ((P*)sd.dgamma)[d] = (P)(float)s;
    }
}

int qr_check(const iseg_qk_norm_rope_geom* g)
{
    if (!g || !is_float_dtype(g->dtype) || !is_float_dtype(g->p_dtype) ||
        (g->pos_dtype != ISEG_I32 && g->pos_dtype != ISEG_I64) || g->pairs < 0 || g->pairs > 1 || g->norm < 0 ||
        g->norm > 1 || !(g->eps >= 0.f && g->eps <= 3.4028234e38f) || !(fabsf(g->mscale) <= 3.4028234e38f))
        return ISEG_ERR_ARG;
    if (g->T < 0 || g->T >= (int64_t)1 << 31 || g->Hq < 0 || g->Hk < 0 || g->D < 1 || g->rope_dim < 0 || g->rope_dim > g->D ||
        g->rope_dim % 2)
        return ISEG_ERR_SHAPE;
    if ((g->Hq > 0 && (g->q_ld < 0 || g->q_hs < 0)) || (g->Hk > 0 && (g->k_ld < 0 || g->k_hs < 0))) return ISEG_ERR_SHAPE;
    return g->D <= 512 && g->Hq <= 65536 && g->Hk <= 65536 ? ISEG_OK : ISEG_ERR_UNSUPPORTED;
}

// tokens of a block's turn: about 128 rows, whose table fits, and blocks for
// the whole card from few tokens
void qr_deal(const iseg_qk_norm_rope_geom* g, int64_t H, bool bwd, int32_t* tokens, int32_t* blocks)
{
    *tokens = 0;
    *blocks = 0;
    if (H < 1 || g->T < 1) return;
    int64_t t = 128 / H;
    const int64_t half = g->rope_dim / 2;
    if (half > 0 && t > kTableMax / half) t = kTableMax / half;
    if (t > g->T / 512) t = g->T / 512;
    if (t < 1) t = 1;
    int64_t b = ceil_div64(g->T, t);
    const int64_t most = bwd ? kBwdBlocks : kRowGridMax;
    *tokens = (int32_t)t;
    *blocks = (int32_t)(b < most ? b : most);
}

template <typename T, typename P, int N, int LPR, int SPL, bool BWD>
int qr_launch(const QrArgs& a, hipStream_t s)
{
    const int b = a.side[0].blocks > a.side[1].blocks ? a.side[0].blocks : a.side[1].blocks;
    if (b > 0) hipLaunchKernelGGL((k_qk_norm_rope<T, P, N, LPR, SPL, BWD>), dim3((unsigned)b, 2), dim3(256), 0, s, a);
    if (BWD && (a.side[0].dgamma || a.side[1].dgamma))
        hipLaunchKernelGGL((k_qk_dgamma<P>), dim3((unsigned)ceil_div64(a.D, 16), 2), dim3(1024), 0, s, a);
    return launch_ok();
}

// whole 16-byte vectors where the rotated part and the row are made of them,
// single elements otherwise
template <typename T, typename P, bool BWD>
int qr_dispatch(const QrArgs& a, hipStream_t s)
{
    constexpr int N = 16 / (int)sizeof(T);
    if (a.D % N == 0 && a.R % (a.pairs ? N : 2 * N) == 0) {
        const int halves = a.pairs ? 0 : a.R / (2 * N);
        const int slots = halves + (int)ceil_div64(a.D - halves * 2 * N, 2 * N);
        if (slots <= 4) return qr_launch<T, P, N, 4, 1, BWD>(a, s);
        if (slots <= 8) return qr_launch<T, P, N, 8, 1, BWD>(a, s);
        if (slots <= 16) return qr_launch<T, P, N, 16, 1, BWD>(a, s);
        if (slots <= 32) return qr_launch<T, P, N, 32, 1, BWD>(a, s);
        return qr_launch<T, P, N, 64, 1, BWD>(a, s);
    }
    const int slots = (a.D + 1) / 2;
    if (slots <= 64) return qr_launch<T, P, 1, 64, 1, BWD>(a, s);
    if (slots <= 128) return qr_launch<T, P, 1, 64, 2, BWD>(a, s);
    return qr_launch<T, P, 1, 64, 4, BWD>(a, s);
}

template <bool BWD>
int qr_types(int32_t dtype, int32_t p_dtype, const QrArgs& a, hipStream_t s)
{
    switch (dtype * 8 + p_dtype) {
    case ISEG_F32 * 8 + ISEG_F32: return qr_dispatch<float, float, BWD>(a, s);
    case ISEG_F32 * 8 + ISEG_F16: return qr_dispatch<float, f16_t, BWD>(a, s);
    case ISEG_F32 * 8 + ISEG_BF16: return qr_dispatch<float, bf16_t, BWD>(a, s);
    case ISEG_F16 * 8 + ISEG_F32: return qr_dispatch<f16_t, float, BWD>(a, s);
    case ISEG_F16 * 8 + ISEG_F16: return qr_dispatch<f16_t, f16_t, BWD>(a, s);
    case ISEG_F16 * 8 + ISEG_BF16: return qr_dispatch<f16_t, bf16_t, BWD>(a, s);
    case ISEG_BF16 * 8 + ISEG_F32: return qr_dispatch<bf16_t, float, BWD>(a, s);
    case ISEG_BF16 * 8 + ISEG_F16: return qr_dispatch<bf16_t, f16_t, BWD>(a, s);
    default: return qr_dispatch<bf16_t, bf16_t, BWD>(a, s);
    }
}

QrArgs qr_args(const iseg_qk_norm_rope_geom* g, const void* q, const void* k, const void* positions,
               const float* inv_freq, const void* gamma_q, const void* gamma_k, bool bwd)
{
    QrArgs a = {};
    a.side[0].x = q; a.side[0].gamma = g->norm ? gamma_q : nullptr; a.side[0].H = g->Hq;
    a.side[0].x_ld = g->q_ld; a.side[0].x_hs = g->q_hs;
    a.side[1].x = k; a.side[1].gamma = g->norm ? gamma_k : nullptr; a.side[1].H = g->Hk;
    a.side[1].x_ld = g->k_ld; a.side[1].x_hs = g->k_hs;
    for (int i = 0; i < 2; i++) qr_deal(g, a.side[i].H, bwd, &a.side[i].tokens, &a.side[i].blocks);
    a.pos = positions; a.freq = inv_freq; a.T = g->T; a.D = (int32_t)g->D; a.R = g->rope_dim; a.pairs = g->pairs;
    a.norm = g->norm; a.pos64 = g->pos_dtype == ISEG_I64; a.eps = g->eps; a.mscale = g->mscale;
    return a;
}

}  // namespace

extern "C" int iseg_qk_norm_rope_fwd(const void* q, const void* k, const void* positions, const float* inv_freq,
                                     const void* gamma_q, const void* gamma_k, const iseg_qk_norm_rope_geom* g,
                                     void* yq, void* yk, int32_t* dev_status, hipStream_t stream)
{
    const int rc = qr_check(g);
    if (rc != ISEG_OK) return rc;
    if (!rows_apart(g->T, g->Hq, g->D, g->yq_ld, g->yq_hs) || !rows_apart(g->T, g->Hk, g->D, g->yk_ld, g->yk_hs))
        return ISEG_ERR_SHAPE;
    if (g->T == 0 || (g->Hq == 0 && g->Hk == 0)) return ISEG_OK;
    if ((g->Hq > 0 && (!q || !yq)) || (g->Hk > 0 && (!k || !yk)) || (g->rope_dim > 0 && (!positions || !inv_freq)))
        return ISEG_ERR_ARG;
    QrArgs a = qr_args(g, q, k, positions, inv_freq, gamma_q, gamma_k, false);
    a.side[0].out = yq; a.side[0].o_ld = g->yq_ld; a.side[0].o_hs = g->yq_hs;
    a.side[1].out = yk; a.side[1].o_ld = g->yk_ld; a.side[1].o_hs = g->yk_hs;
    a.status = dev_status;
    return qr_types<false>(g->dtype, g->p_dtype, a, stream);
}

extern "C" size_t iseg_qk_norm_rope_bwd_ws(const iseg_qk_norm_rope_geom* g)
{
    if (qr_check(g) != ISEG_OK) return 0;
    if (!g->norm) return kNoWs;
    int32_t t, b[2];
    qr_deal(g, g->Hq, true, &t, &b[0]);
    qr_deal(g, g->Hk, true, &t, &b[1]);
    return ws_used((size_t)(b[0] + b[1]) * (size_t)g->D * 4);
}

extern "C" int iseg_qk_norm_rope_bwd(const void* dyq, const void* dyk, const void* q, const void* k,
                                     const void* positions, const float* inv_freq, const void* gamma_q,
                                     const void* gamma_k, const iseg_qk_norm_rope_geom* g, void* dq, void* dk,
                                     void* dgamma_q, void* dgamma_k, void* ws, size_t ws_bytes, hipStream_t stream)
{
    const int rc = qr_check(g);
    if (rc != ISEG_OK) return rc;
    if (!rows_apart(g->T, g->Hq, g->D, g->dq_ld, g->dq_hs) || !rows_apart(g->T, g->Hk, g->D, g->dk_ld, g->dk_hs) ||
        (g->Hq > 0 && (g->yq_ld < 0 || g->yq_hs < 0)) || (g->Hk > 0 && (g->yk_ld < 0 || g->yk_hs < 0)))
        return ISEG_ERR_SHAPE;
    if (!g->norm && (dgamma_q || dgamma_k)) return ISEG_ERR_ARG;
    if (g->T > 0 && ((g->Hq > 0 && (!dyq || !dq || (g->norm && !q))) || (g->Hk > 0 && (!dyk || !dk || (g->norm && !k))) ||
                     (g->rope_dim > 0 && (g->Hq > 0 || g->Hk > 0) && (!positions || !inv_freq))))
        return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_qk_norm_rope_bwd_ws(g)) return ISEG_ERR_WORKSPACE;
    QrArgs a = qr_args(g, q, k, positions, inv_freq, gamma_q, gamma_k, true);
    a.side[0].dy = dyq; a.side[0].dy_ld = g->yq_ld; a.side[0].dy_hs = g->yq_hs;
    a.side[0].out = dq; a.side[0].o_ld = g->dq_ld; a.side[0].o_hs = g->dq_hs; a.side[0].dgamma = dgamma_q;
    a.side[1].dy = dyk; a.side[1].dy_ld = g->yk_ld; a.side[1].dy_hs = g->yk_hs;
    a.side[1].out = dk; a.side[1].o_ld = g->dk_ld; a.side[1].o_hs = g->dk_hs; a.side[1].dgamma = dgamma_k;
    if (dgamma_q) a.side[0].part = (float*)ws;
    if (dgamma_k) a.side[1].part = (float*)ws + (int64_t)a.side[0].blocks * g->D;
    return qr_types<true>(g->dtype, g->p_dtype, a, stream);
}
