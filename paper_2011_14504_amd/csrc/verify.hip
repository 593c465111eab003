// verify.hip -- drafted tokens against the target's probabilities
// (iseg_verify_drafts).
//
// Two kernels: in the first every wave decides how many drafts stand (2 S
// gathers, all at once) and sums some pieces of the row that the next token comes
// from; in the second a block per request finds the piece and then the element
// where the running sum passes u times the whole.  (Both in one block of 1024 threads
// per request: 50021 tokens 20 us against 8.5 captured.)  Sums are float64: of float32
// probabilities they are good to 2^-50, so that a random number of 24 bits meets a
// border between tokens by accident about once in 2^26.
#include "rowops.h"

namespace {

constexpr int kPieces = 1024;            // of a row, at most

struct VfArgs {
    const void *target, *draft, *tokens;
    const int32_t* n_draft;
    const float *u, *us;
    int32_t *out, *accepted;
    double* sums;                        // [B][pieces][2]: of the remainder, of the target
    int32_t* said;                       // [B]: twice the accepted drafts, and 1 if one was refused
    int64_t S, V, t_bs, t_ld, d_bs, d_ld;
    int32_t vecs;                        // vectors of a lane in a piece
    int32_t pieces, per_wave, blocks;    // pieces of a row, of a wave, and blocks of a row
    int32_t tok64;
    int32_t* status;
};

__device__ __forceinline__ int64_t vf_token(const VfArgs& a, int64_t b, int64_t i)
{
    const int64_t at = b * a.S + i;
    return a.tok64 ? ((const int64_t*)a.tokens)[at] : (int64_t)((const int32_t*)a.tokens)[at];
}

__device__ __forceinline__ bool odd_value(float v) { return !(v >= 0.f && v <= 3.4028234e38f); }

// drafts of request b that stand, decided by a wave; `refused`: one did not.  Their
// probabilities are looked at here, the refused one's with its row.
template <typename T>
__device__ __forceinline__ int64_t vf_accepted(const VfArgs& a, int64_t b, bool& refused, int& bad)
{
    int64_t n = a.n_draft[b];
    if (n < 0 || n > a.S) { bad |= ISEG_DEV_RANGE; n = n < 0 ? 0 : a.S; }
    const int lane = threadIdx.x & 63;
    refused = false;
    for (int64_t i0 = 0; i0 < n; i0 += 64) {
        const int64_t i = i0 + lane;
        bool no = false, odd = false;
        if (i < n) {
            const int64_t x = vf_token(a, b, i);
            no = true;
            if (x >= 0 && x < a.V) {
                const float p = (float)((const T*)a.target)[b * a.t_bs + i * a.t_ld + x];
                const float q = a.draft ? (float)((const T*)a.draft)[b * a.d_bs + i * a.d_ld + x] : 1.f;
                no = !((double)a.u[b * a.S + i] * (double)q < (double)p);
                odd = odd_value(p) || odd_value(q);
            }
        }
        const uint64_t m = __ballot(no);
        if (__ballot(odd) & ((m & -m) - 1)) bad |= ISEG_DEV_NONFINITE;     // below the first refused, or all
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

// a double moved by DPP, 0 where the pattern reads past its row
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// sum of v over the lanes up to this one
__device__ __forceinline__ double wave_scan_f64(double v)
{
    v += dpp_f64<0x111, 0xf>(v);
    v += dpp_f64<0x112, 0xf>(v);
    v += dpp_f64<0x114, 0xf>(v);
    v += dpp_f64<0x118, 0xf>(v);
    v += dpp_f64<0x142, 0xa>(v);
    return v + dpp_f64<0x143, 0xc>(v);
}

__device__ __forceinline__ double lane63_f64(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// a lane's values from v on: what is left of p, and p itself; those past the row
// are 0
template <typename T>
struct VfVec {
    static constexpr int N = RowVec<T>::N;
    float p[N], q[N];
    __device__ __forceinline__ VfVec(const VfRow<T>& row, int64_t v, int64_t V)
    {
        RowVec<T> x, y;
        if (v + N <= V) {
            x = row_load(row.p + v);
            if (row.q) y = row_load(row.q + v);
        } else {
            const int n = v < V ? (int)(V - v) : 0;
            x = row_load_part(row.p + v, n, (T)0.f);
            if (row.q) y = row_load_part(row.q + v, n, (T)0.f);
        }
#pragma unroll
        for (int i = 0; i < N; i++) {
            p[i] = (float)x.v[i];
            q[i] = row.q ? (float)y.v[i] : (v + i == row.sure ? 1.f : 0.f);
        }
    }
};

// Bound by memory, one row of p and one of q for each request: 64 x 131072 float32,
// 67 MB, in 14.3 to 15.1 us, 4.5 to 4.7 TB/s.  One request: 4 us, the gathers and then
// the row.
template <typename T>
__global__ __launch_bounds__(256) void k_verify_sums(VfArgs a)
{
    constexpr int N = RowVec<T>::N;
    const int64_t b = blockIdx.x / a.blocks;
    const int lane = threadIdx.x & 63, first = ((int)(blockIdx.x % a.blocks) * 4 + (int)(threadIdx.x >> 6)) * a.per_wave;
    int bad = 0;
    bool refused, odd = false;
    const int64_t acc = vf_accepted<T>(a, b, refused, bad);
    const VfRow<T> row = vf_row<T>(a, b, acc, refused);
    if (first == 0 && lane == 0) a.said[b] = (int32_t)(acc * 2 + refused);
    for (int k = first; k < first + a.per_wave && k < a.pieces; k++) {
        double sr = 0.0, sp = 0.0;
        for (int j = 0; j < a.vecs; j++) {
            const VfVec<T> x(row, (((int64_t)k * a.vecs + j) * 64 + lane) * N, a.V);
#pragma unroll
            for (int i = 0; i < N; i++) {
                odd = odd || odd_value(x.p[i]) || odd_value(x.q[i]);
                sr += left_of(x.p[i], x.q[i]);
                sp += (double)x.p[i];
            }
        }
        sr = wave_scan_f64(sr);
        sp = wave_scan_f64(sp);
        if (lane == 63) {
            double* o = a.sums + (b * a.pieces + k) * 2;
            o[0] = sr;
            o[1] = sp;
        }
    }
    if (odd) bad |= ISEG_DEV_NONFINITE;
    if (bad) set_status(a.status, bad);
}

// A block per request: the piece, then the element.  Where u is below 1 the first
// piece whose running sum passes u times the whole has the token; should rounding
// leave none, the last value with any mass is taken.  7.8 us at 64 requests, 5.9 at
// one: a chain of five trips to memory and LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_verify_pick(VfArgs a)
{
    constexpr int N = RowVec<T>::N;
    __shared__ double wsum[4][2], from;
    __shared__ int first, last;
    const int64_t b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t said = a.said[b], acc = said >> 1;
    const VfRow<T> row = vf_row<T>(a, b, acc, said & 1);
    const double* sums = a.sums + b * a.pieces * 2;

    // the pieces: runs of four a thread
    double mine[2][4], pre[2];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int k = (int)threadIdx.x * 4 + i;
        mine[0][i] = k < a.pieces ? sums[2 * k] : 0.0;
        mine[1][i] = k < a.pieces ? sums[2 * k + 1] : 0.0;
    }
#pragma unroll
    for (int c = 0; c < 2; c++) {
        const double s = mine[c][0] + mine[c][1] + mine[c][2] + mine[c][3];
        pre[c] = wave_scan_f64(s);
        if (lane == 63) wsum[wave][c] = pre[c];
        pre[c] -= s;
    }
    if (threadIdx.x == 0) { first = 0x7fffffff; last = -1; }
    __syncthreads();
    const double rest = wsum[0][0] + wsum[1][0] + wsum[2][0] + wsum[3][0];
    const int col = rest > 0.0 ? 0 : 1;                  // the target's row where nothing remains
    const double whole = col ? wsum[0][1] + wsum[1][1] + wsum[2][1] + wsum[3][1] : rest;
    double t = (double)a.us[b] * whole;
    t = t > 0.0 ? t : 0.0;
    {
        double c = col ? pre[1] : pre[0];
        for (int i = 0; i < wave; i++) c += wsum[i][col];
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
        if (hit == first && hit != 0x7fffffff) from = at;
    }
    __syncthreads();
    if (wave == 0) {
        const bool found = first != 0x7fffffff;
        const int piece = found ? first : last;
        t = found ? t - from : __builtin_inf();          // none: the last value with any mass
        int64_t token = -1;
        if (whole > 0.0 && piece >= 0) {
            double base = 0.0;
            for (int j = 0; j < a.vecs; j++) {
                const int64_t v = (((int64_t)piece * a.vecs + j) * 64 + lane) * N;
                const VfVec<T> x(row, v, a.V);
                double w[N], s = 0.0;
#pragma unroll
                for (int i = 0; i < N; i++) {
                    w[i] = col ? (double)x.p[i] : left_of(x.p[i], x.q[i]);
                    s += w[i];
                }
                const double upto = wave_scan_f64(s);
                double c = base + upto - s;
                int hit = -1, end = -1;
#pragma unroll
                for (int i = 0; i < N; i++) {
                    c += w[i];
                    if (w[i] > 0.0) {
                        end = i;
                        if (hit < 0 && c > t) hit = i;
                    }
                }
                // the lowest lane with a hit; the highest with any mass stands in for none
                const uint64_t hits = __ballot(hit >= 0), ends = __ballot(end >= 0);
                if (hits) {
                    const int at = __builtin_ctzll(hits);
                    token = (((int64_t)piece * a.vecs + j) * 64 + at) * N + __builtin_amdgcn_readlane(hit, at);
                    break;
                }
                if (ends) {
                    const int at = 63 - __builtin_clzll(ends);
                    token = (((int64_t)piece * a.vecs + j) * 64 + at) * N + __builtin_amdgcn_readlane(end, at);
                }
                base += lane63_f64(upto);
            }
        }
        if (lane == 0) {
            a.out[b * (a.S + 1) + acc] = (int32_t)token;
            a.accepted[b] = (int32_t)acc;
            if (token < 0) set_status(a.status, ISEG_DEV_RANGE);
        }
    }
    for (int64_t i = threadIdx.x; i <= a.S; i += 256)
        if (i != acc) a.out[b * (a.S + 1) + i] = i < acc ? (int32_t)vf_token(a, b, i) : -1;
}

int vf_check(const iseg_verify_geom* g)
{
    if (!g || !is_float_dtype(g->dtype) || (g->token_dtype != ISEG_I32 && g->token_dtype != ISEG_I64)) return ISEG_ERR_ARG;
    if (g->B < 0 || g->S < 0 || g->V < 1 || g->V >= (int64_t)1 << 31 || g->t_bs < 0 || g->t_ld < 0 || g->d_bs < 0 || g->d_ld < 0)
        return ISEG_ERR_SHAPE;
    return g->B <= 1 << 16 && g->S <= 1 << 20 ? ISEG_OK : ISEG_ERR_UNSUPPORTED;      // a launch's threads
}

// Pieces of a row: 64 vectors each, or a multiple of that in rows of more than
// 1024 of them (what the second kernel takes); a wave sums up to eight where there
// are enough for the whole card.
void vf_deal(const iseg_verify_geom* g, VfArgs* a)
{
    const int64_t n = 64 * (g->dtype == ISEG_F32 ? 4 : 8);
    a->vecs = (int32_t)ceil_div64(g->V, n * kPieces);
    a->pieces = (int32_t)ceil_div64(g->V, n * a->vecs);
    const int64_t per = g->B * a->pieces / 8192;
    a->per_wave = (int32_t)(per < 1 ? 1 : (per > 8 ? 8 : per));
    a->blocks = (int32_t)ceil_div64(a->pieces, 4 * a->per_wave);
}

template <typename T>
int vf_launch(const VfArgs& a, int64_t B, hipStream_t s)
{
    hipLaunchKernelGGL((k_verify_sums<T>), dim3((unsigned)(B * a.blocks)), dim3(256), 0, s, a);
    hipLaunchKernelGGL((k_verify_pick<T>), dim3((unsigned)B), dim3(256), 0, s, a);
    return launch_ok();
}

}  // namespace

extern "C" size_t iseg_verify_drafts_ws(const iseg_verify_geom* g)
{
    if (vf_check(g) != ISEG_OK) return 0;
    VfArgs a = {};
    vf_deal(g, &a);
    return ws_used(align256((size_t)g->B * (size_t)a.pieces * 16) + (size_t)g->B * 4);
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
    vf_deal(g, &a);
    a.said = (int32_t*)((char*)ws + align256((size_t)g->B * a.pieces * 16));
    a.tok64 = g->token_dtype == ISEG_I64; a.status = dev_status;
    return g->dtype == ISEG_F32   ? vf_launch<float>(a, g->B, stream)
           : g->dtype == ISEG_F16 ? vf_launch<f16_t>(a, g->B, stream)
                                  : vf_launch<bf16_t>(a, g->B, stream);
}
