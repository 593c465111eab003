// logprob.hip -- log probabilities of given tokens with the entropy and the
// most likely alternatives of each row, and their gradient.
//
// One pass over a row keeps, per thread, the running maximum m, S = sum
// e^(x-m) and T = sum e^(x-m) (x-m) (in base 2), and which of the thread's
// vectors held its largest value, its leader.  The k largest logits lie in the
// segments (the vectors of one thread) with the k best leaders: a logit of any
// other segment is beaten by k leaders.  So only those segments are read
// again, and of them only what is no worse than the k-th leader is ranked.
#include "rowops.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kMinF32 = -3.4028234e38f;
constexpr int kTopMax = 64;
constexpr int kCand = 512;                 // candidates ranked in LDS at once
constexpr int kMergeKeys = 1024;           // keys of all splits of a row, leaders of all waves

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

// 2^x to one step; results below 2^-126 count as 0
__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// the sums of a part whose maximum is m, relative to the maximum mn >= m
__device__ __forceinline__ void stat_move(Stat& s, float mn)
{
    const float d = fmaxf((s.m - mn) * kLog2e, -200.f);      // 2^-200 is 0 in float32
    const float c = exp2_raw(d);
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

// a wave's 64 parts joined, the same in every lane: one move to the largest
// maximum, then two sums (8192 x 4096 bf16 28.1 us, 30.2 joined pair by pair)
__device__ __forceinline__ Stat wave_stat(Stat s)
{
    float mn = s.m;
    mn = fmaxf(mn, dpp_f32<0x111>(mn, mn));
    mn = fmaxf(mn, dpp_f32<0x112>(mn, mn));
    mn = fmaxf(mn, dpp_f32<0x114>(mn, mn));
    mn = fmaxf(mn, dpp_f32<0x118>(mn, mn));
    mn = fmaxf(mn, dpp_f32<0x142>(mn, mn));
    mn = fmaxf(mn, dpp_f32<0x143>(mn, mn));
    stat_move(s, lane63_f32(mn));
    return Stat{s.m, wave_sum_f32(s.S), wave_sum_f32(s.T)};
}

__device__ __forceinline__ int64_t token_of(const LpArgs& a, int64_t m)
{
    return a.tok64 ? ((const int64_t*)a.tok)[m] : (int64_t)((const int32_t*)a.tok)[m];
}

// the given token of a row and its logit, loaded ahead of the row itself
struct Given {
    int64_t t;
    float x;
};

template <typename T>
__device__ __forceinline__ Given given_of(const LpArgs& a, int64_t m)
{
    const int64_t t = token_of(a, m);
    return {t, t >= 0 && t < a.V ? (float)((const T*)a.x)[m * a.ld + t] : 0.f};
}

// the scalars of a row from its statistics
__device__ __forceinline__ void row_scalars(const LpArgs& a, int64_t m, const Stat& s, const Given& given)
{
    const int64_t t = given.t;
    float lse, ent, lp;
    if (s.S == 0.f) {                                        // every logit is -infinity
        lse = -__builtin_inff();
        ent = 0.f;
        lp = -__builtin_inff();
    } else {
        const float ls = logf(s.S);
        lse = s.m + ls;
        ent = ls - s.T * kLn2 / s.S;
        lp = given.x - s.m - ls;
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

// how many of the n keys (n a multiple of 4, zeros behind the last) beat `mine`
__device__ __forceinline__ int rank_of(const uint64_t* keys, int n, uint64_t mine)
{
    int r = 0;
#pragma unroll 4
    for (int i = 0; i < n; i += 4) {
        const ulonglong2 a = *(const ulonglong2*)(keys + i), b = *(const ulonglong2*)(keys + i + 2);
        r += (a.x > mine) + (a.y > mine) + (b.x > mine) + (b.y > mine);
    }
    return r;
}

// Ranks the keys held one per thread (0: none) and hands the k best to
// put(rank, key, thread): each wave's k-th best bounds the k-th best of all
// from below, so only the keys at or above the largest of these bounds (a few
// more than k, as a rule) are ranked against each other.  keys: 256 words,
// list: 260, bound: one word per wave, count: one int, all LDS; every thread of
// the block of 256 calls it.
template <typename F>
__device__ __forceinline__ void best_keys(uint64_t mine, int k, uint64_t* keys, uint64_t* list, uint16_t* who,
                                          uint64_t* bound, int* count, F put)
{
    const int tid = threadIdx.x, w = tid >> 6;
    keys[tid] = mine;
    if (tid == 0) *count = 0;
    if ((tid & 63) == 0) bound[w] = 0;
    __syncthreads();
    if (mine && rank_of(keys + w * 64, 64, mine) == k - 1) bound[w] = mine;      // keys differ: one lane at most
    __syncthreads();
    uint64_t lo = 1;
#pragma unroll
    for (int i = 0; i < 4; i++) lo = bound[i] > lo ? bound[i] : lo;
    if (mine >= lo) {
        const int at = atomicAdd(count, 1);
        list[at] = mine;
        who[at] = (uint16_t)tid;
    }
    __syncthreads();
    const int n = *count, n4 = (n + 3) & ~3;
    if (tid < n4 - n) list[n + tid] = 0;
    __syncthreads();
    if (tid < n) {
        const uint64_t key = list[tid];
        const int r = rank_of(list, n4, key);
        if (r < k) put(r, key, who[tid]);
    }
    __syncthreads();
}

// the exponentials of U vectors, to whose largest logit s has been moved
template <typename T, bool ENT, int U>
__device__ __forceinline__ void lp_take(const RowVec<T>* r, Stat& s)
{
    constexpr int N = RowVec<T>::N;
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float d = ((float)r[u].v[i] - s.m) * kLog2e;
            const float e = exp2_raw(d);
            s.S += e;
            if (ENT) s.T = fmaf(e, fmaxf(d, -200.f), s.T);
        }
}

template <typename T>
__device__ __forceinline__ float vec_max(const RowVec<T>& r)
{
    float cm = (float)r.v[0];
#pragma unroll
    for (int i = 1; i < RowVec<T>::N; i++) cm = fmaxf(cm, (float)r.v[i]);
    return cm;
}

// A block's part of a row.  fp32 is bound by memory: 2048 x 50021 with entropy
// and 5 alternatives 80 us, 5.1 TB/s.  16-bit logits are bound by the
// issue of 12 vector instructions for each, one of them an exponential that takes
// four slots (15 with alternatives; counted at 4096 x 32768): 2048 x 50021 bf16 61
// us with 5 alternatives, 54 without (3.8 TB/s), 4096 x 32768 60 (4.5 TB/s).  4 x 131072
// bf16 in 32 parts with 20 alternatives 8.5 us, bound by latency.
// Six waves per SIMD where alternatives are ranked hide more of the ranking's
// latency (1957 x 13910 fp16, 20 of them, 25.8 us; 28 with the four that the
// registers of four open vectors leave); without them it gains nothing.
template <typename T, bool ENT, bool TOP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(TOP ? 6 : 1))) void k_logprob_fwd(LpArgs a)
{
    constexpr int N = RowVec<T>::N, NT = 256, NW = 4, U = 4;
    __shared__ Stat rstat[NW];
    __shared__ __attribute__((aligned(16))) uint64_t keys[TOP ? NT : 1];
    __shared__ __attribute__((aligned(16))) uint64_t cand[TOP ? kCand + 4 : 1];
    __shared__ uint64_t bound[NW];
    __shared__ uint16_t who[TOP ? NT : 1];
    __shared__ int sel[TOP ? kTopMax : 1];
    __shared__ int count;
    __shared__ uint64_t thr_s;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t G = ceil_div64(a.V, N), Gfull = a.V / N;
    for (int64_t item = blockIdx.x; item < a.M * a.splits; item += gridDim.x) {
        const int64_t m = a.splits == 1 ? item : item / a.splits;
        const int sp = (int)(item - m * a.splits);
        const T* x = (const T*)a.x + m * a.ld;
        const int64_t g0 = G * sp / a.splits, g1 = G * (sp + 1) / a.splits;
        const int64_t gf = g1 < Gfull ? g1 : Gfull;
        Given given = {-1, 0.f};
        if (a.splits == 1 && tid == 0) given = given_of<T>(a, m);
        Stat s = {kMinF32, 0.f, 0.f};
        float best = -__builtin_inff();
        int64_t bestg = g0 + tid;
        int64_t g = g0 + tid;
        for (; g + (U - 1) * NT < gf; g += U * NT) {
            RowVec<T> r[U];
#pragma unroll
            for (int u = 0; u < U; u++) r[u] = row_load(x + (g + u * NT) * N);
            float top = s.m;
#pragma unroll
            for (int u = 0; u < U; u++) {
                const float cm = vec_max(r[u]);
                top = fmaxf(top, cm);
                if (TOP && cm > best) { best = cm; bestg = g + u * NT; }
            }
            stat_move(s, top);
            lp_take<T, ENT, U>(r, s);
        }
        for (; g < gf; g += NT) {
            const RowVec<T> r = row_load(x + g * N);
            const float cm = vec_max(r);
            if (TOP && cm > best) { best = cm; bestg = g; }
            stat_move(s, fmaxf(s.m, cm));
            lp_take<T, ENT, 1>(&r, s);
        }
        if (g < g1) {                         // the row's last, broken vector
            const RowVec<T> r = lp_load(x, g, a.V);
            const float cm = vec_max(r);
            if (TOP && cm > best) { best = cm; bestg = g; }
            stat_move(s, fmaxf(s.m, cm));
            lp_take<T, ENT, 1>(&r, s);
        }
        const bool has = g0 + tid < g1;
        s = wave_stat(s);
        if (lane == 0) rstat[w] = s;
        if (tid == 0) thr_s = 0;
        __syncthreads();
        s = stat_join(stat_join(rstat[0], rstat[1]), stat_join(rstat[2], rstat[3]));
        if (a.splits == 1) {
            if (tid == 0) row_scalars(a, m, s, given);
        } else if (tid == 0) {
            float* p = a.pstat + item * 4;
            p[0] = s.m; p[1] = s.S; p[2] = s.T;
        }
        if (TOP) {
            const int k = a.k;
            const int nthr = (int)(g1 - g0 < NT ? g1 - g0 : NT);         // threads with a segment
            const int nsel = k < nthr ? k : nthr;
            best_keys(has ? key_of(best, (uint32_t)bestg) : 0, nsel, keys, cand, who, bound, &count,
                          [&](int rank, uint64_t key, int t) {
                              sel[rank] = t;
                              // with k segments chosen, nothing below the last leader's value, or of
                              // its value behind its vector, counts
                              if (rank == k - 1)
                                  thr_s = (key >> 32) << 32 | (uint32_t)~(uint32_t)((uint32_t)~(uint32_t)key * (uint32_t)N + N - 1);
                          });
            if (tid == 0) count = 0;
            __syncthreads();
            const uint32_t nit = (uint32_t)ceil_div64(g1 - g0, NT);
            uint64_t lo = thr_s, hi = ~0ull, thr = lo;
            for (;;) {
                // candidates with a key of at least thr; when they are too many
                // (ties, or a sorted row) thr is raised by bisection
                for (uint32_t p = tid; p < (uint32_t)nsel * nit; p += NT) {
                    const uint32_t q = p / nit;
                    const int64_t gg = g0 + sel[q] + (int64_t)NT * (p - q * nit);
                    if (gg >= g1) continue;
                    const RowVec<T> r = lp_load(x, gg, a.V);
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        const int64_t c = gg * N + i;
                        const uint64_t key = key_of((float)r.v[i], (uint32_t)c);
                        if (c < a.V && key >= thr) {
                            const int at = atomicAdd(&count, 1);
                            if (at < kCand) cand[at] = key;
                        }
                    }
                }
                __syncthreads();
                const int n = count;
                __syncthreads();
                if (tid == 0) count = 0;
                if (n > kCand) {
                    lo = thr;
                } else if (n < k && thr != lo) {
                    hi = thr;
                } else {
                    const int n4 = (n + 3) & ~3;
                    if (tid < n4 - n) cand[n + tid] = 0;
                    __syncthreads();
                    for (int q = tid; q < n; q += NT) {
                        const uint64_t mk = cand[q];
                        const int rk = rank_of(cand, n4, mk);
                        if (rk >= k) continue;
                        if (a.splits == 1) write_top(a, m, rk, mk, s);
                        else a.pkey[item * k + rk] = mk;
                    }
                    // fewer than k: a short split, or a row with NaN in it
                    for (int q = n + tid; q < k; q += NT) {
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

// Joins the splits of a row.  Each split's keys are in order, so the first
// ceil(k / splits) of every split hold k keys, and the k-th best of these
// bounds the k-th best of all from below; what is at or above it is ranked.  4
// rows of 32 parts with 20 keys each 4.8 us, bound by the latency of its steps.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void k_logprob_join(LpArgs a)
{
    constexpr int PER = kMergeKeys / 256;
    __shared__ __attribute__((aligned(16))) uint64_t list[TOP ? kMergeKeys + 4 : 1];
    __shared__ unsigned long long bound;
    __shared__ int count;
    const int tid = threadIdx.x;
    const int k = a.k, n = a.splits * k;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const uint64_t* key = a.pkey + m * n;
        uint64_t mine[PER];
#pragma unroll
        for (int i = 0; i < PER; i++) mine[i] = TOP && tid + i * 256 < n ? key[tid + i * 256] : 0;
        Given given = {-1, 0.f};
        if (tid == 0) given = given_of<T>(a, m);
        // every wave joins the statistics for itself: its lanes take the splits
        Stat s = {kMinF32, 0.f, 0.f};
        for (int i = tid & 63; i < a.splits; i += 64) {
            const float* p = a.pstat + (m * a.splits + i) * 4;
            s = stat_join(s, Stat{p[0], p[1], p[2]});
        }
        s = wave_stat(s);
        if (tid == 0) row_scalars(a, m, s, given);
        if (TOP) {
            const int j = (k + a.splits - 1) / a.splits, h = j * a.splits, h4 = (h + 3) & ~3;
            if (tid == 0) { bound = 1; count = 0; }
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int e = tid + i * 256, sp = e / k, r = e - sp * k;
                if (e < n && r < j) list[sp * j + r] = mine[i];
            }
            if (tid < h4 - h) list[h + tid] = 0;
            __syncthreads();
            for (int q = tid; q < h; q += 256)
                if (list[q] && rank_of(list, h4, list[q]) == k - 1) bound = list[q];      // keys differ: one at most
            __syncthreads();
            const uint64_t lo = bound;
#pragma unroll
            for (int i = 0; i < PER; i++)
                if (mine[i] >= lo) list[atomicAdd(&count, 1)] = mine[i];
            __syncthreads();
            const int c = count, c4 = (c + 3) & ~3;
            if (tid < c4 - c) list[c + tid] = 0;
            __syncthreads();
            for (int q = tid; q < c; q += 256) {
                const uint64_t mk = list[q];
                const int rk = rank_of(list, c4, mk);
                if (rk < k) write_top(a, m, rk, mk, s);
            }
            for (int q = c + tid; q < k; q += 256) write_none(a, m, q);
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

// what a row's logits are measured from: log p = (x - hi) - lo
struct LbBase {
    float hi, lo;
};

template <typename T, bool H>
__device__ __forceinline__ RowVec<T> lb_take(const RowVec<T>& r, LbBase b, float ent, float glp, float gh, int at)
{
    constexpr int N = RowVec<T>::N;
    RowVec<T> o;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float lp = ((float)r.v[i] - b.hi) - b.lo;
        const float p = exp2_raw(lp * kLog2e);
        const float d = -p * (H ? fmaf(gh, fmaxf(lp, -200.f) + ent, glp) : glp);
        o.v[i] = (T)(i == at ? d + glp : d);
    }
    return o;
}

// float32 holds lse to 2^-25 of its size, and what it lost there is a factor of
// every p: all of log V where a row is filled with its type's lowest value.  From
// 256 on (a loss above 2^-17) the block sums the row again and takes its largest
// logit and the log of the sum apart, unless lse is not this row's (that of a
// vocabulary of which these are a part, say): then e^(x - lse) is what is asked
// for.  Logits below that, a model's as a rule, are read once (4096 x 32768 bf16
// 93.5 us; 178 with every row at 300).
constexpr float kLbFar = 256.f;

template <typename T>
__device__ __forceinline__ LbBase lb_far(const T* x, int64_t V, float lse, Stat* rstat)
{
    const int64_t G = ceil_div64(V, RowVec<T>::N);
    Stat s = {kMinF32, 0.f, 0.f};
    for (int64_t g = threadIdx.x; g < G; g += 256) {
        const RowVec<T> r = lp_load(x, g, V);
        stat_move(s, fmaxf(s.m, vec_max(r)));
        lp_take<T, false, 1>(&r, s);
    }
    s = wave_stat(s);
    __syncthreads();                          // rstat may still be read for the row before
    if ((threadIdx.x & 63) == 0) rstat[threadIdx.x >> 6] = s;
    __syncthreads();
    s = stat_join(stat_join(rstat[0], rstat[1]), stat_join(rstat[2], rstat[3]));
    const float ls = logf(s.S);
    // the forward's lse is off by its own rounding, at most 2^-24 of it, and by
    // what a sum in another order differs by
    return fabsf((s.m - lse) + ls) <= fmaf(1.1920929e-7f, fabsf(lse), 6.1035156e-5f) ? LbBase{s.m, ls} : LbBase{lse, 0.f};
}

constexpr int kLbVecs = 2048;              // vectors of a row per block: eight per thread, four at once

// Bound by memory, logits read and the gradient written once: 4096 x 32768 bf16
// 93.7 us (5.7 TB/s).

template <typename T, bool H>
__global__ __launch_bounds__(256) void k_logprob_bwd(LbArgs a, uint32_t cblocks)
{
    constexpr int N = RowVec<T>::N, U = 4;
    __shared__ Stat rstat[4];
    const int64_t G = ceil_div64(a.V, N), Gfull = a.V / N;
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
        // a row of banned tokens only: every probability, and the gradient, is 0
        const bool empty = lse == -__builtin_inff();
        const float glp = a.g_lp && t >= 0 && !empty ? a.g_lp[m] : 0.f;
        const float gh = H && !empty ? a.g_h[m] : 0.f;
        const float ent = H && !empty ? a.entropy[m] : 0.f;
        LbBase base = {empty ? 0.f : lse, 0.f};
        if (fabsf(lse) >= kLbFar && fabsf(lse) <= 3.4028234e38f) base = lb_far(x, a.V, lse, rstat);
        const int64_t tg = t < 0 ? -1 : t / N;
        const int ti = t < 0 ? -1 : (int)(t - tg * N);
        const int64_t g1 = (cb + 1) * kLbVecs < G ? (cb + 1) * kLbVecs : G;
        const int64_t gf = g1 < Gfull ? g1 : Gfull;
        int64_t g = cb * kLbVecs + threadIdx.x;
        for (; g + (U - 1) * 256 < gf; g += U * 256) {
            RowVec<T> r[U];
#pragma unroll
            for (int u = 0; u < U; u++) r[u] = row_load(x + (g + u * 256) * N);
#pragma unroll
            for (int u = 0; u < U; u++)
                row_store(dx + (g + u * 256) * N, lb_take<T, H>(r[u], base, ent, glp, gh, g + u * 256 == tg ? ti : -1));
        }
        for (; g < gf; g += 256)
            row_store(dx + g * N, lb_take<T, H>(row_load(x + g * N), base, ent, glp, gh, g == tg ? ti : -1));
        if (g < g1)
            row_store_part(dx + g * N, lb_take<T, H>(lp_load(x, g, a.V), base, ent, glp, gh, g == tg ? ti : -1),
                           (int)(a.V - g * N));
    }
}

// Splits of a row: a CU alone takes in about 20 GB/s, so with few rows each is
// cut, down to two vectors per thread (eight with more than 16 rows, which
// fill the chip by themselves sooner), at the cost of a second kernel that
// joins the parts.  4 x 131072 bf16 without alternatives: one block of sixteen
// waves per row 16.2 us, 32 parts and their join 7.2 us.
int lp_splits(const iseg_logprob_geom* g)
{
    const int64_t G = ceil_div64(g->V, g->dtype == ISEG_F32 ? 4 : 8);
    const int64_t fill = 1024 / (g->M > 0 ? g->M : 1);
    const int64_t most = G / (g->M <= 16 ? 512 : 2048);
    int64_t s = most < fill ? most : fill;
    const int64_t cap = g->top_k > 4 ? kMergeKeys / g->top_k : 256;
    s = s < cap ? s : cap;
    return (int)(s > 1 ? s : 1);
}

int lp_check(const iseg_logprob_geom* g)
{
    if (!g || !is_float_dtype(g->dtype) || g->reserved) return ISEG_ERR_ARG;
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
    if (a.k > 0 && a.entropy) hipLaunchKernelGGL((k_logprob_fwd<T, true, true>), grid, dim3(256), 0, s, a);
    else if (a.k > 0) hipLaunchKernelGGL((k_logprob_fwd<T, false, true>), grid, dim3(256), 0, s, a);
    else if (a.entropy) hipLaunchKernelGGL((k_logprob_fwd<T, true, false>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_logprob_fwd<T, false, false>), grid, dim3(256), 0, s, a);
    if (a.splits > 1) {
        const dim3 jgrid((unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax));
        if (a.k > 0) hipLaunchKernelGGL((k_logprob_join<T, true>), jgrid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_logprob_join<T, false>), jgrid, dim3(256), 0, s, a);
    }
    return launch_ok();
}

template <typename T>
int launch_bwd(const LbArgs& a, hipStream_t s)
{
    const int64_t cblocks = ceil_div64(ceil_div64(a.V, RowVec<T>::N), kLbVecs);
    const int64_t items = a.M * cblocks;
    const dim3 grid((unsigned)(items < kRowGridMax ? items : kRowGridMax));
    if (a.g_h) hipLaunchKernelGGL((k_logprob_bwd<T, true>), grid, dim3(256), 0, s, a, (uint32_t)cblocks);
    else hipLaunchKernelGGL((k_logprob_bwd<T, false>), grid, dim3(256), 0, s, a, (uint32_t)cblocks);
    return launch_ok();
}

}  // namespace

extern "C" size_t iseg_logprob_fwd_ws(const iseg_logprob_geom* g)
{
    if (lp_check(g) != ISEG_OK) return 0;
    const size_t sp = (size_t)lp_splits(g);
    if (sp == 1 || g->M == 0) return kNoWs;
    return ws_used(align256((size_t)g->M * sp * 16) + align256((size_t)g->M * sp * (size_t)g->top_k * 8));
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
