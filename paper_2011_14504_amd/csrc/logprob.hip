// logprob.hip -- log probabilities of given tokens with the entropy and the
// most likely alternatives of each row, and their gradient.
//
// One pass over a row keeps, per thread, the running maximum m, S = sum
// e^(x-m) and T = sum e^(x-m) (x-m) (in base 2), and which of the thread's
// vectors held its largest value.  The k largest logits lie in the segments
// (the vectors of one thread) with the k best leaders, so only those segments
// are read again.
#include "rowops.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kMinF32 = -3.4028234e38f;
constexpr int kTopMax = 64;
constexpr int kCand = 512;                 // candidates ranked in LDS at once
constexpr int kMergeKeys = 1024;           // keys of all splits of a row

struct LpArgs {
    const void *x, *tok;
    float *logprob, *lse, *entropy, *tlp;
    int32_t* ids;
    float* pstat;                // [M][splits][4] m, S, T
    uint64_t* pkey;              // [M][splits][k]
    int64_t M, V, ld;
    int32_t k, splits, tok64;
    int32_t* status;
};

// an order of floats as an order of unsigned integers (-0 counts as 0, a NaN
// as the least value)
__device__ __forceinline__ uint32_t ord_of(float v)
{
    if (v != v) return 0;
    const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float of_ord(uint32_t o)
{
    return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// larger key = better: larger value, then lower index; 0 = none
__device__ __forceinline__ uint64_t key_of(float v, uint32_t idx) { return (uint64_t)ord_of(v) << 32 | (uint32_t)~idx; }

struct Stat {
    float m, S, T;
};

// weight of a part whose maximum is m when the maximum is mn (and its exponent)
__device__ __forceinline__ void stat_move(Stat& s, float mn)
{
    const float d = fmaxf((s.m - mn) * kLog2e, -200.f);      // 2^-200 is 0 in float32
    const float c = exp2f(d);
    s.T = c * fmaf(s.S, d, s.T);
    s.S *= c;
    s.m = mn;
}

__device__ __forceinline__ Stat stat_join(Stat a, Stat b)
{
    const float mn = fmaxf(a.m, b.m);
    stat_move(a, mn);
    stat_move(b, mn);
    return Stat{mn, a.S + b.S, a.T + b.T};
}

__device__ __forceinline__ int64_t token_of(const LpArgs& a, int64_t m)
{
    return a.tok64 ? ((const int64_t*)a.tok)[m] : (int64_t)((const int32_t*)a.tok)[m];
}

// the scalars of a row from its statistics
template <typename T>
__device__ __forceinline__ void row_scalars(const LpArgs& a, int64_t m, const Stat& s)
{
    const int64_t t = token_of(a, m);
    float lse, ent, lp;
    if (s.S == 0.f) {                                        // every logit is -infinity
        lse = -__builtin_inff();
        ent = 0.f;
        lp = -__builtin_inff();
    } else {
        const float ls = logf(s.S);
        lse = s.m + ls;
        ent = ls - s.T * kLn2 / s.S;
        lp = t >= 0 && t < a.V ? (float)((const T*)a.x)[m * a.ld + t] - s.m - ls : 0.f;
        if (!(s.S == s.S)) {
            lse = ent = lp = s.S;
            set_status(a.status, ISEG_DEV_NONFINITE);
        }
    }
    if (t >= a.V) {
        lp = __builtin_nanf("");
        set_status(a.status, ISEG_DEV_RANGE);
    }
    a.logprob[m] = t < 0 ? 0.f : lp;
    a.lse[m] = lse;
    if (a.entropy) a.entropy[m] = ent;
}

__device__ __forceinline__ void write_top(const LpArgs& a, int64_t m, int rank, uint64_t key, const Stat& s)
{
    const float v = of_ord((uint32_t)(key >> 32));
    a.ids[m * a.k + rank] = (int32_t)~(uint32_t)key;
    a.tlp[m * a.k + rank] = s.S == 0.f ? -__builtin_inff() : !(s.S == s.S) ? s.S : v - s.m - logf(s.S);
}

__device__ __forceinline__ void write_none(const LpArgs& a, int64_t m, int rank)
{
    a.ids[m * a.k + rank] = 0;
    a.tlp[m * a.k + rank] = __builtin_nanf("");
}

// one vector of a row, -infinity past the row's end
template <typename T>
__device__ __forceinline__ RowVec<T> lp_load(const T* x, int64_t g, int64_t V)
{
    constexpr int N = RowVec<T>::N;
    const int64_t c = g * N;
    if (c + N <= V) return row_load(x + c);
    return row_load_part(x + c, (int)(V - c), (T)-__builtin_inff());
}

template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprob_fwd(LpArgs a)
{
    constexpr int N = RowVec<T>::N;
    __shared__ Stat rstat[4];
    __shared__ uint64_t keys[TOP ? 256 : 1];
    __shared__ uint64_t cand[TOP ? kCand : 1];
    __shared__ int sel[TOP ? kTopMax : 1];
    __shared__ int ncand;
    __shared__ uint64_t thr_s;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t G = ceil_div64(a.V, N);
    for (int64_t item = blockIdx.x; item < a.M * a.splits; item += gridDim.x) {
        const int64_t m = item / a.splits;
        const int sp = (int)(item - m * a.splits);
        const T* x = (const T*)a.x + m * a.ld;
        const int64_t g0 = G * sp / a.splits, g1 = G * (sp + 1) / a.splits;
        Stat s = {kMinF32, 0.f, 0.f};
        float best = -__builtin_inff();
        int64_t bestg = g0 + tid;
        for (int64_t g = g0 + tid; g < g1; g += 256) {
            const RowVec<T> r = lp_load(x, g, a.V);
            float cm = (float)r.v[0];
#pragma unroll
            for (int i = 1; i < N; i++) cm = fmaxf(cm, (float)r.v[i]);
            if (TOP && cm > best) { best = cm; bestg = g; }
            stat_move(s, fmaxf(s.m, cm));
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float d = ((float)r.v[i] - s.m) * kLog2e;
                const float e = exp2f(d);
                s.S += e;
                s.T = fmaf(e, fmaxf(d, -200.f), s.T);
            }
        }
        const bool has = g0 + tid < g1;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            Stat t = {__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.T, o, 64)};
            s = stat_join(s, t);
        }
        if (lane == 0) rstat[w] = s;
        if (TOP) keys[tid] = has ? key_of(best, (uint32_t)bestg) : 0;
        if (tid == 0) { ncand = 0; thr_s = 0; }
        __syncthreads();
        s = rstat[0];
#pragma unroll
        for (int i = 1; i < 4; i++) s = stat_join(s, rstat[i]);
        if (a.splits == 1) {
            if (tid == 0) row_scalars<T>(a, m, s);
        } else if (tid == 0) {
            float* p = a.pstat + item * 4;
            p[0] = s.m; p[1] = s.S; p[2] = s.T;
        }
        if (TOP) {
            const int k = a.k;
            const int nthr = (int)(g1 - g0 < 256 ? g1 - g0 : 256);       // threads with a segment
            const int nsel = k < nthr ? k : nthr;
            const uint64_t mine = keys[tid];
            int rank = 0;
            for (int i = 0; i < 256; i++) rank += keys[i] > mine;
            if (has && rank < nsel) {
                sel[rank] = tid;
                // with k segments chosen, nothing below the last one's leader counts
                if (rank == k - 1) thr_s = (mine >> 32) << 32 | (uint32_t)~(uint32_t)((int64_t)(uint32_t)~(uint32_t)mine * N + N - 1);
            }
            __syncthreads();
            const int64_t nit = ceil_div64(g1 - g0, 256);
            uint64_t lo = thr_s, hi = ~0ull, thr = lo;
            for (;;) {
                // candidates with a key of at least thr
                for (int64_t p = tid; p < nsel * nit; p += 256) {
                    const int64_t g = g0 + sel[p / nit] + 256 * (p % nit);
                    if (g >= g1) continue;
                    const RowVec<T> r = lp_load(x, g, a.V);
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        const int64_t c = g * N + i;
                        const uint64_t key = key_of((float)r.v[i], (uint32_t)c);
                        if (c < a.V && key >= thr) {
                            const int at = atomicAdd(&ncand, 1);
                            if (at < kCand) cand[at] = key;
                        }
                    }
                }
                __syncthreads();
                const int n = ncand;
                __syncthreads();
                if (tid == 0) ncand = 0;
                if (n > kCand) lo = thr;
                else if (n < k && thr != lo) hi = thr;
                else {
                    for (int q = tid; q < n; q += 256) {
                        const uint64_t mk = cand[q];
                        int rk = 0;
                        for (int i = 0; i < n; i++) rk += cand[i] > mk;
                        if (rk >= k) continue;
                        if (a.splits == 1) write_top(a, m, rk, mk, s);
                        else a.pkey[item * k + rk] = mk;
                    }
                    // fewer than k: a short split, or a row with NaN in it
                    for (int q = n + tid; q < k; q += 256) {
                        if (a.splits == 1) write_none(a, m, q);
                        else a.pkey[item * k + q] = 0;
                    }
                    break;
                }
                thr = lo + (hi - lo) / 2;
                __syncthreads();
            }
        }
        __syncthreads();
    }
}

// joins the splits of a row
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprob_join(LpArgs a)
{
    __shared__ uint64_t keys[TOP ? kMergeKeys : 1];
    const int tid = threadIdx.x;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        Stat s = {kMinF32, 0.f, 0.f};
        for (int i = 0; i < a.splits; i++) {
            const float* p = a.pstat + (m * a.splits + i) * 4;
            s = stat_join(s, Stat{p[0], p[1], p[2]});
        }
        if (tid == 0) row_scalars<T>(a, m, s);
        if (TOP) {
            const int n = a.splits * a.k;
            for (int q = tid; q < n; q += 256) keys[q] = a.pkey[m * n + q];
            __syncthreads();
            for (int q = tid; q < n; q += 256) {
                const uint64_t mk = keys[q];
                if (!mk) continue;
                int rk = 0;
                for (int i = 0; i < n; i++) rk += keys[i] > mk;
                if (rk < a.k) write_top(a, m, rk, mk, s);
            }
            int have = 0;
            if (tid < a.k)
                for (int i = 0; i < n; i++) have += keys[i] != 0;
            if (tid < a.k && tid >= have) write_none(a, m, tid);
            __syncthreads();
        }
    }
}

struct LbArgs {
    const void *x, *tok;
    const float *lse, *entropy, *g_lp, *g_h;
    void* dx;
    int64_t M, V, ld, out_ld;
    int32_t tok64;
    int32_t* status;
};

template <typename T>
__global__ __launch_bounds__(256) void k_logprob_bwd(LbArgs a, int64_t cblocks)
{
    constexpr int N = RowVec<T>::N;
    const int64_t G = ceil_div64(a.V, N);
    for (int64_t item = blockIdx.x; item < a.M * cblocks; item += gridDim.x) {
        const int64_t m = item / cblocks;
        const int64_t cb = item - m * cblocks;
        const T* x = (const T*)a.x + m * a.ld;
        T* dx = (T*)a.dx + m * a.out_ld;
        int64_t t = a.tok64 ? ((const int64_t*)a.tok)[m] : (int64_t)((const int32_t*)a.tok)[m];
        if (t >= a.V) {
            if (cb == 0 && threadIdx.x == 0) set_status(a.status, ISEG_DEV_RANGE);
            t = -1;
        }
        const float lse = a.lse[m];
        const bool empty = lse == -__builtin_inff();
        const float glp = a.g_lp && t >= 0 ? a.g_lp[m] : 0.f;
        const float gh = a.g_h ? a.g_h[m] : 0.f;
        const float ent = a.g_h ? a.entropy[m] : 0.f;
        for (int64_t g = cb * 1024 + threadIdx.x; g < (cb + 1) * 1024 && g < G; g += 256) {
            const RowVec<T> r = lp_load(x, g, a.V);
            RowVec<T> o;
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float lp = (float)r.v[i] - lse;
                const float p = exp2f(lp * kLog2e);
                float d = -p * fmaf(gh, fmaxf(lp, -200.f) + ent, glp);
                if (g * N + i == t) d += glp;
                o.v[i] = (T)(empty ? 0.f : d);
            }
            const int64_t c = g * N;
            if (c + N <= a.V) row_store(dx + c, o);
            else row_store_part(dx + c, o, (int)(a.V - c));
        }
    }
}

// splits of a row: enough blocks for the chip when there are few rows, each
// with at least 1024 vectors
int lp_splits(const iseg_logprob_geom* g)
{
    const int64_t n = g->dtype == ISEG_F32 ? 4 : 8;
    const int64_t G = ceil_div64(g->V, n);
    int64_t s = ceil_div64(1024, g->M > 0 ? g->M : 1);
    const int64_t most = G / 1024 > 1 ? G / 1024 : 1;
    s = s < most ? s : most;
    const int64_t cap = g->top_k > 0 ? kMergeKeys / g->top_k : 256;
    s = s < cap ? s : cap;
    return (int)(s > 1 ? s : 1);
}

int lp_check(const iseg_logprob_geom* g)
{
    if (!g || !is_float_dtype(g->dtype)) return ISEG_ERR_ARG;
    if (g->token_dtype != ISEG_I32 && g->token_dtype != ISEG_I64) return ISEG_ERR_ARG;
    if (g->M < 0 || g->V < 1 || g->V >= (int64_t)1 << 31 || g->ld < g->V) return ISEG_ERR_SHAPE;
    if (g->top_k < 0 || g->top_k > kTopMax || g->top_k > g->V) return ISEG_ERR_ARG;
    return ISEG_OK;
}

template <typename T>
int launch_fwd(const LpArgs& a, hipStream_t s)
{
    const int64_t items = a.M * a.splits;
    const dim3 grid((unsigned)(items < kRowGridMax ? items : kRowGridMax));
    const dim3 jgrid((unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax));
    if (a.k > 0) hipLaunchKernelGGL((k_logprob_fwd<T, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_logprob_fwd<T, false>), grid, dim3(256), 0, s, a);
    if (a.splits > 1) {
        if (a.k > 0) hipLaunchKernelGGL((k_logprob_join<T, true>), jgrid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_logprob_join<T, false>), jgrid, dim3(256), 0, s, a);
    }
    return launch_ok();
}

template <typename T>
int launch_bwd(const LbArgs& a, hipStream_t s)
{
    const int64_t cblocks = ceil_div64(ceil_div64(a.V, RowVec<T>::N), 1024);
    const int64_t items = a.M * cblocks;
    hipLaunchKernelGGL(k_logprob_bwd<T>, dim3((unsigned)(items < kRowGridMax ? items : kRowGridMax)), dim3(256), 0, s,
                       a, cblocks);
    return launch_ok();
}

}  // namespace

extern "C" size_t iseg_logprob_fwd_ws(const iseg_logprob_geom* g)
{
    if (lp_check(g) != ISEG_OK) return 0;
    const size_t sp = (size_t)lp_splits(g);
    if (sp == 1 || g->M == 0) return 256;
    return align256((size_t)g->M * sp * 16) + align256((size_t)g->M * sp * (size_t)g->top_k * 8);
}

extern "C" int iseg_logprob_fwd(const void* logits, const void* tokens, const iseg_logprob_geom* g, float* logprob,
                                float* lse, float* entropy, int32_t* top_ids, float* top_logprob, void* ws,
                                size_t ws_bytes, int32_t* dev_status, hipStream_t stream)
{
    const int rc = lp_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->M == 0) return ISEG_OK;
    if (!logits || !tokens || !logprob || !lse || (g->top_k > 0 && (!top_ids || !top_logprob))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_logprob_fwd_ws(g)) return ISEG_ERR_WORKSPACE;
    LpArgs a = {};
    a.x = logits; a.tok = tokens; a.logprob = logprob; a.lse = lse; a.entropy = entropy;
    a.ids = top_ids; a.tlp = top_logprob;
    a.M = g->M; a.V = g->V; a.ld = g->ld; a.k = g->top_k; a.splits = lp_splits(g);
    a.tok64 = g->token_dtype == ISEG_I64; a.status = dev_status;
    a.pstat = (float*)ws;
    a.pkey = (uint64_t*)((char*)ws + align256((size_t)g->M * a.splits * 16));
    return g->dtype == ISEG_F32 ? launch_fwd<float>(a, stream)
                                : g->dtype == ISEG_F16 ? launch_fwd<f16_t>(a, stream) : launch_fwd<bf16_t>(a, stream);
}

extern "C" int iseg_logprob_bwd(const void* logits, const void* tokens, const float* lse, const float* entropy,
                                const float* g_logprob, const float* g_entropy, const iseg_logprob_geom* g,
                                void* dlogits, int32_t* dev_status, hipStream_t stream)
{
    const int rc = lp_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->out_ld < g->V) return ISEG_ERR_SHAPE;
    if (g->M == 0) return ISEG_OK;
    if ((!g_logprob && !g_entropy) || (g_entropy && !entropy)) return ISEG_ERR_ARG;
    if (!logits || !tokens || !lse || !dlogits) return ISEG_ERR_ARG;
    LbArgs a = {};
    a.x = logits; a.tok = tokens; a.lse = lse; a.entropy = entropy; a.g_lp = g_logprob; a.g_h = g_entropy;
    a.dx = dlogits; a.M = g->M; a.V = g->V; a.ld = g->ld; a.out_ld = g->out_ld;
    a.tok64 = g->token_dtype == ISEG_I64; a.status = dev_status;
    return g->dtype == ISEG_F32 ? launch_bwd<float>(a, stream)
                                : g->dtype == ISEG_F16 ? launch_bwd<f16_t>(a, stream) : launch_bwd<bf16_t>(a, stream);
}
