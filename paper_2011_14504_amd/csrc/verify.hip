// verify.hip -- drafted tokens against the target's probabilities
// (iseg_verify_drafts).
//
// Two kernels: the first decides how many drafts stand (every block for itself:
// 2 S gathers) and sums one part of the row that the next token comes from; the
// second finds the part and then the element where the running sum passes u
// times the whole.  Sums are float64: of float32 probabilities they are good to
// 2^-50, so that a random number of 24 bits meets a border between tokens by
// accident about once in 2^26.
#include "rowops.h"

namespace {

constexpr int kParts = 1024;             // of a row, at most
constexpr int kPartMin = 2048;           // elements of a part, at least

struct VfArgs {
    const void *target, *draft, *tokens;
    const int32_t* n_draft;
    const float *u, *us;
    int32_t *out, *accepted;
    double* sums;                        // [B][parts][2]: of the remainder, of the target
    int32_t* said;                       // [B]: twice the accepted drafts, and 1 if one was refused
    int64_t S, V, t_bs, t_ld, d_bs, d_ld, part;
    int32_t parts, tok64;
    int32_t* status;
};

__device__ __forceinline__ int64_t vf_token(const VfArgs& a, int64_t b, int64_t i)
{
    const int64_t at = b * a.S + i;
    return a.tok64 ? ((const int64_t*)a.tokens)[at] : (int64_t)((const int32_t*)a.tokens)[at];
}

// drafts of request b that stand, decided by a wave; `refused`: one did not
template <typename T>
__device__ __forceinline__ int64_t vf_accepted(const VfArgs& a, int64_t b, bool& refused, int& bad)
{
    int64_t n = a.n_draft[b];
    if (n < 0 || n > a.S) { bad |= ISEG_DEV_RANGE; n = n < 0 ? 0 : a.S; }
    const int lane = threadIdx.x & 63;
    refused = false;
    for (int64_t i0 = 0; i0 < n; i0 += 64) {
        const int64_t i = i0 + lane;
        bool no = false;
        if (i < n) {
            const int64_t x = vf_token(a, b, i);
            no = true;
            if (x >= 0 && x < a.V) {
                const double p = (double)(float)((const T*)a.target)[b * a.t_bs + i * a.t_ld + x];
                const double q = a.draft ? (double)(float)((const T*)a.draft)[b * a.d_bs + i * a.d_ld + x] : 1.0;
                no = !((double)a.u[b * a.S + i] * q < p);
            }
        }
        const uint64_t m = __ballot(no);
        if (m) {
            const int64_t i = i0 + __builtin_ctzll(m), x = vf_token(a, b, i);
            if (x < 0 || x >= a.V) bad |= ISEG_DEV_RANGE;
            refused = true;
            return i;
        }
    }
    return n;
}

// the row that the next token comes from
template <typename T>
struct VfRow {
    const T *p, *q;                      // q: NULL where nothing is taken off, or the draft was certain
    int64_t sure;                        // the certain draft, or -1
};

template <typename T>
__device__ __forceinline__ VfRow<T> vf_row(const VfArgs& a, int64_t b, int64_t acc, bool refused)
{
    VfRow<T> r = {(const T*)a.target + b * a.t_bs + acc * a.t_ld, nullptr, -1};
    if (refused) {
        if (a.draft) r.q = (const T*)a.draft + b * a.d_bs + acc * a.d_ld;
        else r.sure = vf_token(a, b, acc);
    }
    return r;
}

__device__ __forceinline__ double left_of(float p, float q)
{
    const double d = (double)p - (double)q;
    return d > 0.0 ? d : 0.0;
}

__device__ __forceinline__ bool odd_value(float v) { return !(v >= 0.f && v <= 3.4028234e38f); }

__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void k_verify_sums(VfArgs a)
{
    constexpr int N = RowVec<T>::N;
    __shared__ double red[2][4];
    const int64_t b = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    int bad = 0;
    bool refused, odd = false;
    const int64_t acc = vf_accepted<T>(a, b, refused, bad);
    const VfRow<T> row = vf_row<T>(a, b, acc, refused);
    const int64_t v0 = part * a.part, v1 = v0 + a.part < a.V ? v0 + a.part : a.V;
    double sr = 0.0, sp = 0.0;
    int64_t v = v0 + (int64_t)threadIdx.x * N;
    for (; v + N <= v1; v += 256 * N) {
        const RowVec<T> p = row_load(row.p + v);
        RowVec<T> q;
        if (row.q) q = row_load(row.q + v);
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float pf = (float)p.v[i], qf = row.q ? (float)q.v[i] : (v + i == row.sure ? 1.f : 0.f);
            odd = odd || odd_value(pf) || odd_value(qf);
            sr += left_of(pf, qf);
            sp += (double)pf;
        }
    }
    for (; v < v1; v++) {                          // one thread's short vector
        const float pf = (float)row.p[v], qf = row.q ? (float)row.q[v] : (v == row.sure ? 1.f : 0.f);
        odd = odd || odd_value(pf) || odd_value(qf);
        sr += left_of(pf, qf);
        sp += (double)pf;
    }
    if (odd) bad |= ISEG_DEV_NONFINITE;
    if (bad) set_status(a.status, bad);
    if (part == 0 && threadIdx.x == 0) a.said[b] = (int32_t)(acc * 2 + refused);
    sr = wave_sum_f64(sr);
    sp = wave_sum_f64(sp);
    if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = sr; red[1][threadIdx.x >> 6] = sp; }
    __syncthreads();
    if (threadIdx.x < 2) {
        const double* r = red[threadIdx.x];
        a.sums[(b * a.parts + part) * 2 + threadIdx.x] = r[0] + r[1] + r[2] + r[3];
    }
}

// sum of v over the lanes up to this one
__device__ __forceinline__ double wave_scan_f64(double v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(v, o, 64);
        if (lane >= o) v += t;
    }
    return v;
}

// A block per request: the part, then the element.  Where u is below 1 the first
// part whose running sum passes u times the whole has the token; should rounding
// leave none, the last value with any mass is taken.
template <typename T>
__global__ __launch_bounds__(256) void k_verify_pick(VfArgs a)
{
    constexpr int N = RowVec<T>::N, K = 32 / N;          // vectors of a thread in a turn of 8192 values
    __shared__ double total[2], from[4], seg[4][K];
    __shared__ int first, last;
    const int64_t b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t said = a.said[b], acc = said >> 1;
    const VfRow<T> row = vf_row<T>(a, b, acc, said & 1);
    const double* sums = a.sums + b * a.parts * 2;
    int bad = 0;

    // the parts: runs of four a thread
    double mine[2][4], pre[2];
#pragma unroll
    for (int c = 0; c < 2; c++) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = (int)threadIdx.x * 4 + i;
            mine[c][i] = k < a.parts ? sums[2 * k + c] : 0.0;
            s += mine[c][i];
        }
        pre[c] = wave_scan_f64(s);
        if (lane == 63) seg[wave][c] = pre[c];
        pre[c] -= s;
    }
    if (threadIdx.x == 0) { first = 0x7fffffff; last = -1; }
    __syncthreads();
    if (threadIdx.x < 2) total[threadIdx.x] = seg[0][threadIdx.x] + seg[1][threadIdx.x] + seg[2][threadIdx.x] + seg[3][threadIdx.x];
    __syncthreads();
    const int col = total[0] > 0.0 ? 0 : 1;              // the target's row where nothing remains
    double t = (double)a.us[b] * total[col];
    t = t > 0.0 ? t : 0.0;
    {
        double c = col ? pre[1] : pre[0];
        for (int i = 0; i < wave; i++) c += seg[i][col];
        int hit = 0x7fffffff, pos = -1;
        double at = 0.0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const double w = col ? mine[1][i] : mine[0][i];
            const int k = (int)threadIdx.x * 4 + i;
            if (w > 0.0) {
                pos = k;
                if (hit == 0x7fffffff && c + w > t) { hit = k; at = c; }
            }
            c += w;
        }
        if (hit != 0x7fffffff) atomicMin(&first, hit);
        if (pos >= 0) atomicMax(&last, pos);
        __syncthreads();
        if (hit == first && hit != 0x7fffffff) from[0] = at;
    }
    __syncthreads();
    const int64_t part = first != 0x7fffffff ? first : last;
    t = first != 0x7fffffff ? t - from[0] : __builtin_inf();
    const bool any = total[col] > 0.0 && part >= 0;
    __syncthreads();
    if (threadIdx.x == 0) { first = 0x7fffffff; last = -1; }

    // the element: turns of 8192 values, a quarter a wave, in vectors; the sums of
    // a wave's 64 N values first, then the lanes of the one that passes t
    int64_t token = -1;
    if (any) {
        const int64_t v0 = part * a.part, v1 = v0 + a.part < a.V ? v0 + a.part : a.V;
        double base = 0.0;
        int pos = -1;                                    // this thread's last value with any mass
        for (int64_t s0 = v0; s0 < v1; s0 += 8192) {
            double w[K][N], s[K];
#pragma unroll
            for (int k = 0; k < K; k++) {
                const int64_t v = s0 + ((int64_t)(wave * K + k) * 64 + lane) * N;
                RowVec<T> p, q;
                if (v + N <= v1) {
                    p = row_load(row.p + v);
                    if (row.q) q = row_load(row.q + v);
                } else {
                    const int n = v < v1 ? (int)(v1 - v) : 0;
                    p = row_load_part(row.p + v, n, (T)0.f);
                    if (row.q) q = row_load_part(row.q + v, n, (T)0.f);
                }
                s[k] = 0.0;
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const float pf = (float)p.v[i], qf = row.q ? (float)q.v[i] : (v + i == row.sure ? 1.f : 0.f);
                    w[k][i] = col ? (double)pf : left_of(pf, qf);
                    s[k] += w[k][i];
                    if (w[k][i] > 0.0) pos = (int)(v + i - v0);
                }
            }
#pragma unroll
            for (int k = 0; k < K; k++) {
                const double x = wave_sum_f64(s[k]);
                if (lane == 0) seg[wave][k] = x;
            }
            __syncthreads();
            double c = base;
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int k = 0; k < K; k++) {
                    const double x = seg[i][k];
                    if (i == wave && c <= t && c + x > t) {          // at most one piece
                        double e = c + wave_scan_f64(s[k]) - s[k];
                        int hit = 0x7fffffff, end = -1;
                        const int at = (int)(s0 - v0) + ((wave * K + k) * 64 + lane) * N;
#pragma unroll
                        for (int n = 0; n < N; n++) {
                            e += w[k][n];
                            if (w[k][n] > 0.0) {
                                end = at + n;
                                if (hit == 0x7fffffff && e > t) hit = at + n;
                            }
                        }
                        // rounding may leave none: then its last value
                        if (__any(hit != 0x7fffffff)) {
                            if (hit != 0x7fffffff) atomicMin(&first, hit);
                        } else {
                            const uint32_t top = wave_top_u32((uint32_t)(end + 1));
                            if (lane == 0 && top) atomicMin(&first, (int)top - 1);
                        }
                    }
                    c += x;
                }
            base = c;
            __syncthreads();
            if (first != 0x7fffffff) break;
        }
        if (pos >= 0) atomicMax(&last, pos);
        __syncthreads();
        const int at = first != 0x7fffffff ? first : last;
        token = at >= 0 ? v0 + at : -1;
    }
    if (token < 0) bad |= ISEG_DEV_RANGE;
    for (int64_t i = threadIdx.x; i <= a.S; i += 256)
        a.out[b * (a.S + 1) + i] = i < acc ? (int32_t)vf_token(a, b, i) : (i == acc ? (int32_t)token : -1);
    if (threadIdx.x == 0) {
        a.accepted[b] = (int32_t)acc;
        if (bad) set_status(a.status, bad);
    }
}

int vf_check(const iseg_verify_geom* g)
{
    if (!g || !is_float_dtype(g->dtype) || (g->token_dtype != ISEG_I32 && g->token_dtype != ISEG_I64)) return ISEG_ERR_ARG;
    if (g->B < 0 || g->S < 0 || g->V < 1 || g->V >= (int64_t)1 << 31 || g->t_bs < 0 || g->t_ld < 0 || g->d_bs < 0 || g->d_ld < 0)
        return ISEG_ERR_SHAPE;
    return g->B <= 1 << 20 && g->S <= 1 << 20 ? ISEG_OK : ISEG_ERR_UNSUPPORTED;
}

// elements of a part: parts for the whole card, each of some length, and no
// more of them than the second kernel deals out
int64_t vf_part(const iseg_verify_geom* g)
{
    const int64_t want = ceil_div64(1024, g->B > 0 ? g->B : 1);
    int64_t part = ceil_div64(g->V, want);
    if (part < kPartMin) part = kPartMin;
    if (part < ceil_div64(g->V, kParts)) part = ceil_div64(g->V, kParts);
    return ceil_div64(part, 256) * 256;
}

template <typename T>
int vf_launch(const VfArgs& a, int64_t B, hipStream_t s)
{
    hipLaunchKernelGGL((k_verify_sums<T>), dim3((unsigned)(B * a.parts)), dim3(256), 0, s, a);
    hipLaunchKernelGGL((k_verify_pick<T>), dim3((unsigned)B), dim3(256), 0, s, a);
    return launch_ok();
}

}  // namespace

extern "C" size_t iseg_verify_drafts_ws(const iseg_verify_geom* g)
{
    if (vf_check(g) != ISEG_OK) return 0;
    return ws_used(align256((size_t)g->B * (size_t)ceil_div64(g->V, vf_part(g)) * 16) + (size_t)g->B * 4);
}

extern "C" int iseg_verify_drafts(const void* target, const void* draft, const void* tokens, const int32_t* n_draft,
                                  const float* u, const float* u_sample, const iseg_verify_geom* g, int32_t* out,
                                  int32_t* accepted, void* ws, size_t ws_bytes, int32_t* dev_status, hipStream_t stream)
{
    const int rc = vf_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->B == 0) return ISEG_OK;
    if (!target || !n_draft || !u_sample || !out || !accepted || (g->S > 0 && (!tokens || !u))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_verify_drafts_ws(g)) return ISEG_ERR_WORKSPACE;
    VfArgs a = {};
    a.target = target; a.draft = draft; a.tokens = tokens; a.n_draft = n_draft; a.u = u; a.us = u_sample;
    a.out = out; a.accepted = accepted; a.sums = (double*)ws;
    a.S = g->S; a.V = g->V; a.t_bs = g->t_bs; a.t_ld = g->t_ld; a.d_bs = g->d_bs; a.d_ld = g->d_ld;
    a.part = vf_part(g);
    a.parts = (int32_t)ceil_div64(g->V, a.part);
    a.said = (int32_t*)((char*)ws + align256((size_t)g->B * a.parts * 16));
    a.tok64 = g->token_dtype == ISEG_I64; a.status = dev_status;
    return g->dtype == ISEG_F32   ? vf_launch<float>(a, g->B, stream)
           : g->dtype == ISEG_F16 ? vf_launch<f16_t>(a, g->B, stream)
                                  : vf_launch<bf16_t>(a, g->B, stream);
}
