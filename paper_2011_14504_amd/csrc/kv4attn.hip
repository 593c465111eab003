// kv4attn.hip -- attention over the paged 4-bit cache (iseg_kv4_attention).
//
// Rows are the queries of one key head: row r of a request is query r / G, head
// r % G of the G query heads that share it.  A wave takes 16 R rows and steps
// over 32 keys at a time:
//   S^T = K Q^T   on 16x16x32 float16 MFMAs, the codes as A: their scales are a
//                 factor per row of S^T;
//   p = 2^(s - m) with m a whole number 8 to 9 above the running maximum of a row,
//                 moved only when a score passes it; l += p;
//   O^T += V^T P^T, P in the registers that S^T left it in.  V's scale goes into
//                 p, and a power of two of the row's own (`up`) brings the largest
//                 product that the row has seen into float16's range, moved only
//                 when it must be.
// Codes become float16 by placing them in the mantissa of 1024 (9 instructions
// for 8 codes); the layout of the cache makes a lane's operands whole words.
#include "kv4.h"

namespace {

typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef float f2_t __attribute__((ext_vector_type(2)));
typedef float f4_t __attribute__((ext_vector_type(4)));

constexpr float kNone = -3.0e38f;        // m of a row that has seen no key
constexpr float kRoom = 8.f;             // m is whole and above the running maximum by this to one more
constexpr float kTop = 32768.f;          // weights times scale times up are at most this, float16's largest is 65504
constexpr int kUpLog = 10, kUpMost = 100;    // up brings a new largest below 2^10, and is 2^100 at most
constexpr int kQLog = 15;                // queries that are not float16 are brought below 2^15
constexpr int kSplitsMax = 128;

struct KaArgs {
    const void* q;
    const uint8_t *kc, *vc;
    const float *ks, *vs;
    const int32_t *table, *q_start, *kv_len;
    void* out;
    float *lse, *pm, *po;                // parts: (m, l) and rows of W floats
    int64_t T, q_ld, q_hs, o_ld, o_hs, table_ld, n_pages, max_pages, max_q, max_kv, window;
    uint64_t p16_inv;                    // 2^36 / p16, rounded up
    int32_t B, Hq, H, G, D, W, p16;      // p16: tiles of 16 tokens of a page
    int32_t splits, tiles, dtype, causal;
    int32_t join_rows;                   // rows of a tile that may be there
    int32_t rows_min, rows_max;          // rows of the requests that this launch takes: (min, max]
    float scale;                         // times log2 e
    double scale_left;                   // the same before it was rounded, over it
    int32_t* status;
};

// (w & mask) | 1024.0 in both halves, in one instruction: from registers, since
// it takes one literal and these are two
__device__ __forceinline__ h2_t in_1024(uint32_t w, uint32_t mask)
{
    uint32_t k = 0x64006400u;
    asm("" : "+s"(mask), "+v"(k));
    return __builtin_bit_cast(h2_t, (w & mask) | k);
}

// eight float16 of a word of K: codes n + 8 in nibbles 0 4 1 5 (and 2 6 3 7 above)
__device__ __forceinline__ h2_t codes_lo(uint32_t w)
{
    const h2_t k = {(_Float16)1032.f, (_Float16)1032.f};
    return in_1024(w, 0x000f000fu) - k;
}

__device__ __forceinline__ h2_t codes_hi(uint32_t w)
{
    const h2_t s = {(_Float16)0.0625f, (_Float16)0.0625f}, k = {(_Float16)-72.f, (_Float16)-72.f};
    return __builtin_elementwise_fma(in_1024(w, 0x00f000f0u), s, k);
}

// what a float16 leaves of the float32 it was rounded from: v - h[HALF], in one step
template <int HALF>
__device__ __forceinline__ float rest_of(float v, h2_t h)
{
    float r;
    if constexpr (HALF == 0) asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(v));
    else asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(v));
    return r;
}

__device__ __forceinline__ h8_t join8(h2_t a, h2_t b, h2_t c, h2_t d)
{
    return h8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float max4(float v)        // over the four lanes of a row
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

__device__ __forceinline__ float sum4(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

struct KaSeq {
    int64_t q0;                          // first row of q
    int64_t n;                           // its queries
    int64_t kv;                          // keys
};

__device__ __forceinline__ KaSeq ka_seq(const KaArgs& a, int64_t b, int& bad)
{
    KaSeq s;
    s.q0 = a.q_start[b];
    s.n = (int64_t)a.q_start[b + 1] - s.q0;
    s.kv = a.kv_len[b];
    if (s.q0 < 0 || s.n < 0 || s.q0 + s.n > a.T) { bad = 1; s.n = 0; }
    if (s.n > a.max_q) { bad = 1; s.n = 0; }                     // its tiles are not among the launch's
    if (s.kv < 0) { bad = 1; s.kv = 0; }
    if (s.kv > a.max_kv) { bad = 1; s.kv = a.max_kv; }
    return s;
}

// What a block works on: rows row0 .. of a request.  Requests of at most
// rows_max and more than rows_min rows count; with one tile per request tile is
// the request, otherwise their tiles of TR rows follow one another, each
// request's last (its longest) first.
template <int TR, bool SHARED>
__device__ __forceinline__ bool ka_tile(const KaArgs& a, int tile, KaSeq& s, int64_t& b, int64_t& row0, int& bad)
{
    if (SHARED) {
        b = tile;
        s = ka_seq(a, b, bad);
        row0 = 0;
        const int64_t rows = s.n * a.G;
        return rows > a.rows_min && rows <= a.rows_max;
    }
    const int lane = threadIdx.x & 63;
    int64_t base = 0;
    for (int32_t b0 = 0; b0 < a.B; b0 += 64) {
        int64_t tl = 0;
        if (b0 + lane < a.B) {
            const KaSeq t = ka_seq(a, b0 + lane, bad);
            const int64_t rows = t.n * a.G;
            tl = rows > a.rows_min && rows <= a.rows_max ? (rows + TR - 1) / TR : 0;
        }
        int64_t sum = tl;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t v = __shfl_up(sum, o, 64);
            if (lane >= o) sum += v;
        }
        const uint64_t m = __ballot(base + sum > tile);
        if (m) {
            const int at = __builtin_ctzll(m);
            // uniform, and to be seen as such: branches on them are scalar
            const int32_t back = __builtin_amdgcn_readfirstlane((int32_t)(base + __shfl(sum, at, 64) - 1 - tile));
            b = b0 + at;
            int ignored = 0;
            s = ka_seq(a, b, ignored);
            row0 = (int64_t)back * TR;
            return true;
        }
        base += __shfl(sum, 63, 64);
    }
    return false;
}

// keys [lo, hi) that row r of a request sees
__device__ __forceinline__ void ka_span(const KaArgs& a, const KaSeq& s, int64_t r, int64_t& lo, int64_t& hi)
{
    const int64_t pos = s.kv - s.n + r / a.G;
    hi = a.causal && pos + 1 < s.kv ? pos + 1 : s.kv;
    lo = a.window > 0 ? pos + 1 - a.window : 0;
    hi = hi < 0 ? 0 : hi;
    lo = lo < 0 ? 0 : lo;
}

// four elements of an output row that starts at element `at`, from d on: o times
// the inverse of l
__device__ __forceinline__ void ka_store(const KaArgs& a, int64_t at, int d, f4_t o, float inv)
{
    at += d;
    o *= inv;
    if (a.dtype == ISEG_F32) {
        __builtin_memcpy((float*)a.out + at, &o, 16);
    } else if (a.dtype == ISEG_F16) {
        _Float16 x[4] = {(_Float16)o[0], (_Float16)o[1], (_Float16)o[2], (_Float16)o[3]};
        __builtin_memcpy((_Float16*)a.out + at, x, 8);
    } else {
        __bf16 x[4] = {(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
        __builtin_memcpy((__bf16*)a.out + at, x, 8);
    }
}

// 1 / l; 0 for a row without keys
__device__ __forceinline__ float ka_inv(float l) { return l > 0.f ? 1.f / l : (l == l ? 0.f : l); }

// log sum of a row, in float64 and with what the scale's rounding left off: it is the
// whole score's
__device__ __forceinline__ float ka_lse(const KaArgs& a, float m, float l)
{
    if (!(l > 0.f || l != l)) return -__builtin_inff();
    return (float)(((double)m * a.scale_left + log2((double)l)) * 0.693147180559945309);
}

// Where row r of a tile goes: its place among the parts, or its output row.
struct KaOut {
    int64_t at;                          // part, or first element of the output row
    float inv;                           // outputs: 1 / l
};

// `one`: this thread writes the row's m and l, or its lse
template <int TR>
__device__ __forceinline__ KaOut ka_row(const KaArgs& a, const KaSeq& s, int tile, int h, int split, int64_t row0, int r, float m, float l,
                                        bool one)
{
    KaOut o;
    if (a.splits > 1) {
        o.at = (((int64_t)tile * a.H + h) * TR + r) * a.splits + split;
        o.inv = 0.f;
        if (one) { a.pm[o.at * 2] = m; a.pm[o.at * 2 + 1] = l; }
    } else {
        const int64_t q = (row0 + r) / a.G, tok = s.q0 + q, head = h * a.G + (row0 + r - q * a.G);
        o.at = tok * a.o_ld + head * a.o_hs;
        o.inv = ka_inv(l);
        if (one && a.lse) a.lse[tok * a.Hq + head] = ka_lse(a, m, l);
    }
    return o;
}

__device__ __forceinline__ void ka_put(const KaArgs& a, const KaOut& o, int d, f4_t v)
{
    if (a.splits > 1) *(f4_t*)(a.po + o.at * a.W + d) = v;
    else if (d < a.D) ka_store(a, o.at, d, v, o.inv);
}

// eight elements of q's row that starts at element `at`, from d on, or zeros
template <int DT>
__device__ __forceinline__ void ka_get8(const KaArgs& a, int64_t at, int d, bool in, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = 0.f;
    if (!in) return;
    if constexpr (DT == ISEG_F32) {
        __builtin_memcpy(f, (const float*)a.q + at + d, 32);
    } else if constexpr (DT == ISEG_F16) {
        _Float16 x[8];
        __builtin_memcpy(x, (const _Float16*)a.q + at + d, 16);
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = (float)x[i];
    } else {
        __bf16 x[8];
        __builtin_memcpy(x, (const __bf16*)a.q + at + d, 16);
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = (float)x[i];
    }
}

// a lane's words of a tile
template <int NC>
struct KaWords {
    uint32_t w[NC];
};

template <int NC>
__device__ __forceinline__ KaWords<NC> words(const uint8_t* p)
{
    KaWords<NC> r;
    __builtin_memcpy(&r, __builtin_assume_aligned(p, NC % 4 == 0 ? 16 : NC % 2 == 0 ? 8 : 4), NC * 4);
    return r;
}

// What a wave keeps of its 16 R rows.  DT: the tensors' type.  A float16 of q or p is
// one rounding of 2^-11: p is two such terms, and q of float32 tensors.  (With one term
// of p, float16 outputs were 1.5 times as far from 64 bits as their own rounding puts
// them, and bfloat16 ones rounded to the other neighbour in one element of fifteen.)
template <int NC, int R, int DT>
struct KaRows {
    static constexpr int NQ = DT == ISEG_F32 ? 2 : 1, NS = 2;
    static constexpr float k_down = DT == ISEG_F16 ? 1.f : 1.f / (1 << kQLog);      // of k's scales, for the queries' 2^15
    h8_t q[NQ][R][NC];                   // queries as B operands
    float cf[R];                         // score per unit of S^T and scale of k
    int32_t lo[R], hi[R];                // keys that a lane's rows see
    int32_t full_lo, full_hi;            // keys that all rows see
    int32_t any_lo, any_hi;              // keys that some row sees
    f4_t acc[R][2 * NC];
    float m[R], l[R];
    float up[R];                         // acc is sums of codes times weight times V's scale times up

    __device__ __forceinline__ void load(const KaArgs& a, const KaSeq& s, int64_t row0, int64_t rows, int h)
    {
        const int lane = threadIdx.x & 63, c = lane & 15, g4 = lane >> 4;
#pragma unroll
        for (int t = 0; t < R; t++) {
            const int64_t r = row0 + t * 16 + c;
            const bool in = r < rows;
            int64_t l0 = 0, h0 = 0;
            if (in) ka_span(a, s, r, l0, h0);
            lo[t] = (int32_t)l0;
            hi[t] = (int32_t)h0;
            const int64_t at = in ? (s.q0 + r / a.G) * a.q_ld + (h * a.G + r % a.G) * a.q_hs : 0;
            auto get = [&](int w, float (&f)[8]) {
                const int d = g4 * 8 * NC + w * 8;
                ka_get8<DT>(a, at, d, in && d < a.D, f);
            };
            // float16 reaches no further than 65504 and 2^-24: rows of the other types
            // are brought below 2^15 by a power of two first, so that elements down to
            // 2^-31 of the largest keep bfloat16's bits (below 1, down to 2^-16)
            int e = 0;
            if (DT != ISEG_F16) {
                float big = 0.f;
#pragma unroll
                for (int w = 0; w < NC; w++) {
                    float f[8];
                    get(w, f);
#pragma unroll
                    for (int i = 0; i < 8; i++) big = fmaxf(big, fabsf(f[i]));
                }
                big = max4(big);
                if (big > 0.f && big <= 3.4028234e38f) (void)frexpf(big, &e);
                e = e < -100 ? -100 : e;
            }
            cf[t] = fmaxf(ldexpf(a.scale, e), 1.17549435e-38f);      // never 0: a masked score is -infinity times this
#pragma unroll
            for (int w = 0; w < NC; w++) {
                float f[8];
                get(w, f);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float x = DT == ISEG_F16 ? f[i] : ldexpf(f[i], kQLog - e);
                    q[0][t][w][i] = (_Float16)x;
                    if constexpr (NQ > 1) q[NQ - 1][t][w][i] = (_Float16)(x - (float)(_Float16)x);
                }
            }
            m[t] = kNone;
            l[t] = 0.f;
            up[t] = ldexpf(1.f, kUpMost);
#pragma unroll
            for (int i = 0; i < 2 * NC; i++) acc[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
        }
        full_lo = full_hi = any_lo = any_hi = 0;
        if (row0 < rows) {
            const int64_t last = (row0 + 16 * R < rows ? row0 + 16 * R : rows) - 1;
            int64_t l0, h0;
            ka_span(a, s, row0, l0, h0);
            any_lo = (int32_t)l0;
            full_hi = (int32_t)h0;
            ka_span(a, s, last, l0, h0);
            full_lo = (int32_t)l0;
            any_hi = (int32_t)h0;
        }
    }

    // The softmax step of NT tiles of 16 keys from key kb on: scores st, the
    // tiles' scales, whether a tile is there (ok).  Leaves the weights as B
    // operands of V^T P^T in the order of V's words (tokens 0 2 1 3).
    template <int NT>
    __device__ __forceinline__ void soften(f4_t (&st)[R][NT], f4_t (&ks)[NT], f4_t (&vs)[NT], const bool (&ok)[NT], int32_t kb,
                                           int32_t kv, h8_t (&pf)[NS][R][NT / 2])
    {
        const int g4 = (threadIdx.x & 63) >> 4;
        bool full = kb >= full_lo && kb + 16 * NT <= full_hi;
#pragma unroll
        for (int i = 0; i < NT; i++) full = full && ok[i];
        if (!full) {
            asm volatile("");            // a branch: as selects these would be done for every step
            // a weight of 0 times any scale has to be 0: scales of v of no key count
            // as 0, and those that are no number go to the scores that see them
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    if (!(vs[i][r] <= 3.4028234e38f)) {
                        vs[i][r] = 0.f;
                        ks[i][r] = __builtin_nanf("");
                    }
                    if (!(ok[i] && kb + 16 * i + 4 * g4 + r < kv)) vs[i][r] = 0.f;
                }
        }
#pragma unroll
        for (int t = 0; t < R; t++)
#pragma unroll
            for (int i = 0; i < NT; i++) st[t][i] *= ks[i];
        if (!full) {
            asm volatile("");
#pragma unroll
            for (int t = 0; t < R; t++)
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        const int32_t j = kb + 16 * i + 4 * g4 + r;
                        if (!(ok[i] && j >= lo[t] && j < hi[t])) st[t][i][r] = -__builtin_inff();
                    }
        }
        float mx[R];
        bool move = false;
#pragma unroll
        for (int t = 0; t < R; t++) {
            mx[t] = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) mx[t] = fmaxf(mx[t], st[t][i][r]);
            move = move || mx[t] * cf[t] > m[t];
        }
        if (__any(move)) {
#pragma unroll
            for (int t = 0; t < R; t++) {
                // what came before gets smaller by 2^d, d whole: up makes good for it as
                // far as it may, so that acc stays as it is and keeps its bits if what
                // passed it has a small value
                const float mn = fmaxf(m[t], ceilf(fmaf(max4(mx[t]), cf[t], kRoom))), d = mn - m[t];
                int e;
                (void)frexpf(up[t], &e);                         // up = 2^(e - 1)
                const float g = fminf(d, (float)(kUpMost + 1 - e)), al = __builtin_amdgcn_exp2f(g - d);
                m[t] = mn;
                l[t] *= __builtin_amdgcn_exp2f(-d);
                up[t] = ldexpf(up[t], (int)g);
                if (__any(al != 1.f)) {
#pragma unroll
                    for (int i = 0; i < 2 * NC; i++) acc[t][i] *= al;
                }
            }
        }
        float top[R];
        bool high = false;
#pragma unroll
        for (int t = 0; t < R; t++) {
            top[t] = 0.f;
#pragma unroll
            for (int i = 0; i < NT; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float v = __builtin_amdgcn_exp2f(fmaf(st[t][i][r], cf[t], -m[t]));
                    l[t] += v;
                    st[t][i][r] = v * vs[i][r];
                    top[t] = fmaxf(top[t], st[t][i][r]);
                }
            high = high || top[t] * up[t] > kTop;
        }
        if (__any(high)) {
#pragma unroll
            for (int t = 0; t < R; t++) {
                const float big = fminf(max4(top[t]), 3.4028234e38f);
                if (!(big * up[t] > kTop)) continue;
                int e;
                (void)frexpf(big, &e);                           // big in [2^(e-1), 2^e)
                const float n = ldexpf(1.f, kUpLog - e), f = n / up[t];
                up[t] = n;
#pragma unroll
                for (int i = 0; i < 2 * NC; i++) acc[t][i] *= f;
            }
        }
#pragma unroll
        for (int t = 0; t < R; t++)
#pragma unroll
            for (int i = 0; i < NT; i++) {
#pragma unroll
                for (int r = 0; r < 2; r++) {
                    f2_t v = {st[t][i][r] * up[t], st[t][i][r + 2] * up[t]};
                    // the product is rounded once for both terms (contracted with one of
                    // them it would not be the same number)
                    asm("" : "+v"(v.x), "+v"(v.y));
                    const h2_t a = __builtin_convertvector(v, h2_t);
                    const h2_t b = __builtin_convertvector((f2_t{rest_of<0>(v.x, a), rest_of<1>(v.y, a)}), h2_t);
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        pf[0][t][i / 2][4 * (i & 1) + 2 * r + j] = a[j];
                        pf[1][t][i / 2][4 * (i & 1) + 2 * r + j] = b[j];
                    }
                }
            }
    }

    template <int NT>
    __device__ __forceinline__ void score(const h8_t kf, int w, int i, f4_t (&st)[R][NT])
    {
#pragma unroll
        for (int t = 0; t < R; t++)
#pragma unroll
            for (int n = 0; n < NQ; n++) st[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, q[n][t][w], st[t][i], 0, 0, 0);
    }

    // O^T += V^T P^T for columns 16 d .. of a pair of tiles
    template <int NP>
    __device__ __forceinline__ void add(const h8_t vf, int d, int pair, const h8_t (&pf)[NS][R][NP])
    {
#pragma unroll
        for (int t = 0; t < R; t++)
#pragma unroll
            for (int n = 0; n < NS; n++)
                acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[n][t][pair], acc[t][d], 0, 0, 0);
    }
};

// Tiles of 16 tokens that a wave needs, PER a step, STRIDE apart from step to
// step: looked up in the block table for N steps at a time, one lane each, and the
// page ids of the next N steps requested with them.
template <int PER, int STRIDE>
struct KaTiles {
    static constexpr int N = 64 / PER;   // steps of a look-up
    const int32_t* row;
    int32_t first, from, end;            // first tile; those between [from, end) hold keys that a row sees, others are not
                                         // asked for (pages behind a window may be gone)
    int32_t page;                        // of the next look-up
    int idx;                             // -1: past the keys, or a page id out of range
    uint64_t there;                      // idx >= 0
    __device__ __forceinline__ int32_t tile_of(int it) const
    {
        const int lane = threadIdx.x & 63;
        return first + (it + lane / PER) * STRIDE + lane % PER;
    }
    __device__ __forceinline__ int32_t column(const KaArgs& a, int32_t t16) const
    {
        return (int32_t)(((uint64_t)(uint32_t)t16 * a.p16_inv) >> 36);
    }
    __device__ __forceinline__ void ask(const KaArgs& a, int it)
    {
        const int32_t t16 = tile_of(it);
        page = row[t16 < end ? column(a, t16) : 0];
    }
    __device__ __forceinline__ void look(const KaArgs& a, int h, int it)
    {
        const int32_t t16 = tile_of(it), pg = page;
        const bool in = t16 >= from && t16 < end, ok = in && pg >= 0 && pg < a.n_pages;
        if (in && !ok) set_status(a.status, ISEG_DEV_RANGE);
        idx = ok ? (pg * a.H + h) * a.p16 + (t16 - column(a, t16) * a.p16) : -1;
        there = __ballot(ok);
        ask(a, it + N);
    }
    __device__ __forceinline__ int at(int it, int i) const { return __builtin_amdgcn_readlane(idx, (it % N) * PER + i); }
    __device__ __forceinline__ uint32_t mask(int it) const { return (uint32_t)(there >> ((it % N) * PER)) & ((1u << PER) - 1); }
};

// waves per SIMD whose registers the rows leave room for
constexpr int ka_few_waves(int nc, int r, int dt)
{
    const int n = (dt == ISEG_F32 ? 2 : 1) * r * nc;
    return n <= 1 ? 4 : n <= 4 && r < 4 ? 3 : n <= 8 && nc < 8 ? 2 : 1;
}

// ---------------------------------------------------------------------------
// few rows: the four waves of a block hold the same rows and deal the keys among
// themselves
// ---------------------------------------------------------------------------
// Bound by the cache's bytes, each read once: with G = 4 a tile of 16 rows is a quarter
// full and its products cost less than the bytes.  A wave has one step of 32 keys in
// hand and the next one under way, and three waves a SIMD (139 registers; held to four
// waves a call of 64 x 8192 keys takes 154 us, 124 with three) keep about 13 MB on
// their way.  64 requests of 8192 keys, 8 heads of 128: 571 MB in 115 us, 5.0 TB/s, the
// copy's rate.  Shorter work has the blocks' beginnings and ends on top (queries, table
// and first keys one after the other, then the join): 64 of 820 to 8192 keys, 315 MB, 87
// us, of which the loads alone take 72; 1 of 131072, 143 MB, 33 us, the loads 28.  Parts
// dealt by length (prefix sums of all requests in every block) were no faster, and
// slower where all have one length.  float32 tensors: 124 us at 64 x 8192; heads of 256,
// 32 x 8192: 140.  Two and four tiles of rows hold 212 registers and all of them: 16 x
// 8192 with 32 rows 61 us, 64 rows behind 131072 keys 127.
//
// NC: words of a row's quarter (W / 32).  R: tiles of 16 rows.
template <int NC, int R, int DT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(ka_few_waves(NC, R, DT)))) void k_kv4_few(KaArgs a)
{
    constexpr int W = NC * 32, TR = 16 * R;
    __shared__ float so[4 * 16 * (W + 4)];
    __shared__ float sm[4][16], sl[4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g4 = lane >> 4;
    const int h = blockIdx.x % a.H, split = (blockIdx.x / a.H) % a.splits, tile = blockIdx.x / a.H / a.splits;
    int bad = 0;
    KaSeq s;
    int64_t b, row0;
    const bool have = ka_tile<TR, true>(a, tile, s, b, row0, bad);
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
    if (!have) return;
    const int64_t rows = s.n * a.G;
    KaRows<NC, R, DT> x;
    x.load(a, s, 0, rows, h);

    // whole steps of 128 keys, dealt to the splits
    const int32_t k_lo = x.any_lo & ~31, kv = (int32_t)s.kv;
    const int32_t steps = x.any_hi > k_lo ? (x.any_hi - k_lo + 127) / 128 : 0;
    const int32_t per = (steps + a.splits - 1) / a.splits, it0 = split * per;
    const int32_t n_it = it0 + per < steps ? per : (steps > it0 ? steps - it0 : 0);
    const int32_t key0 = k_lo + it0 * 128 + wave * 32;

    // the words of 32 keys; the next step's keys are requested once the scores are
    // there, its values once they are summed up
    KaTiles<2, 8> tl = {a.table + b * a.table_ld, key0 >> 4, x.any_lo >> 4, (kv + 15) >> 4, 0, -1, 0};
    if (n_it > 0) tl.ask(a, 0);
    KaWords<NC> kw[2], vw[2];
    f4_t ks_next[2], vs_next[2];
    auto fetch_k = [&](int it) {
        if (it % tl.N == 0) tl.look(a, h, it);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int ti = tl.at(it, i);
            const int64_t at = ti >= 0 ? ti : 0;
            kw[i] = words<NC>(a.kc + at * (256 * NC) + (c * 4 + g4) * (4 * NC));
            ks_next[i] = *(const f4_t*)(a.ks + at * 16 + g4 * 4);
            vs_next[i] = *(const f4_t*)(a.vs + at * 16 + g4 * 4);
        }
    };
    auto fetch_v = [&](int it) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int ti = tl.at(it, i);
            const int64_t at = ti >= 0 ? ti : 0;
            vw[i] = words<NC>(a.vc + at * (256 * NC) + (c * 4 + g4) * (4 * NC));
        }
    };
    if (n_it > 0) {
        fetch_k(0);
        fetch_v(0);
    }
    for (int it = 0; it < n_it; it++) {
        const int32_t kb = key0 + it * 128;
        if (kb >= x.any_hi) break;
        const uint32_t oks = tl.mask(it);
        const bool ok[2] = {(oks & 1) != 0, (oks & 2) != 0};
        const bool more = it + 1 < n_it;
        f4_t st[R][2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
#pragma unroll
            for (int t = 0; t < R; t++) st[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NC; w++) {
                const uint32_t u = kw[i].w[w], v = u >> 8;
                x.score(join8(codes_lo(u), codes_hi(u), codes_lo(v), codes_hi(v)), w, i, st);
            }
        }
        f4_t ks[2] = {ks_next[0] * x.k_down, ks_next[1] * x.k_down}, vs[2] = {vs_next[0], vs_next[1]};
        if (more) fetch_k(it + 1);
        h8_t pf[x.NS][R][1];
        x.soften(st, ks, vs, ok, kb, kv, pf);
#pragma unroll
        for (int w = 0; w < NC; w++) {
            const uint32_t a0 = vw[0].w[w], a1 = vw[1].w[w], b0 = a0 >> 8, b1 = a1 >> 8;
            x.add(join8(codes_lo(a0), codes_lo(b0), codes_lo(a1), codes_lo(b1)), 2 * w, 0, pf);
            x.add(join8(codes_hi(a0), codes_hi(b0), codes_hi(a1), codes_hi(b1)), 2 * w + 1, 0, pf);
        }
        if (more) fetch_v(it + 1);
    }

    // the waves' rows joined, a tile of 16 at a time: the whole, or this split's part
#pragma unroll
    for (int t = 0; t < R; t++) x.l[t] = sum4(x.l[t]);
    for (int t = 0; t < R; t++) {
        if (t * 16 >= rows) break;
        __syncthreads();
        float* mine = so + (wave * 16 + c) * (W + 4) + g4 * 4;
#pragma unroll
        for (int u = 0; u < R; u++)
            if (u == t) {
#pragma unroll
                for (int i = 0; i < 2 * NC; i++) *(f4_t*)(mine + i * 16) = x.acc[u][i] * (1.f / x.up[u]);
                if (g4 == 0) { sm[wave][c] = x.m[u]; sl[wave][c] = x.l[u]; }
            }
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * (W / 4); e += 256) {
            const int r = e / (W / 4), d = (e - r * (W / 4)) * 4;
            if (t * 16 + r >= rows) continue;
            float mr = sm[0][r];
#pragma unroll
            for (int w = 1; w < 4; w++) mr = fmaxf(mr, sm[w][r]);
            f4_t o = {0.f, 0.f, 0.f, 0.f};
            float lr = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float f = __builtin_amdgcn_exp2f(sm[w][r] - mr);
                o += f * *(const f4_t*)(so + (w * 16 + r) * (W + 4) + d);
                lr += f * sl[w][r];
            }
            ka_put(a, ka_row<TR>(a, s, tile, h, split, 0, t * 16 + r, mr, lr, d == 0), d, o);
        }
    }
}

// ---------------------------------------------------------------------------
// many rows: eight waves with 16 R rows each; 64 keys at a time become float16
// operands in LDS, once for all of them
// ---------------------------------------------------------------------------
// Bound by the sum of matrix and vector instructions: a 16x16x32 product takes 16
// cycles of the matrix cores and 8 of the wave's issue, and a wave does a stage's scores,
// softmax and V's products one after the other, so two waves a SIMD hardly overlap them.
// 3 x 3001 queries behind as many keys, 32 heads over 8 of 128: 1160 to 1200 us for 663
// GFLOP that are needed (550 to 570 TFLOP/s; the library's largest products reach 1377;
// the weights' second term is half as many products again).  Matrix instructions take 400
// of it, the issue of vector instructions 560, the exponentials 100 more.  With one part
// left out: the softmax 760, the products 870, loads and codes to LDS 890.  Loads and
// codes to LDS alone take 600 to 660: a stage's loads are requested one stage ahead and
// wait for memory, which the arithmetic covers.  1 x 4096: 253; in float16 254, in float32
// (two terms of q as well) 351; heads of 256 250.  R = 1 where a request has up to 128
// rows or a prompt is short (ka_cost).
// Tried with one term of the weights, which took 870 to 920, and slower: sixteen waves of
// 16 rows (1158), twelve waves (spills), 32x32x16 products with V's scale per stage (897 to
// 945), stages of 128 keys (896).
constexpr int kWaves = 8;

// a stage of 64 keys: operands of 1 KB each (64 lanes of 16 bytes), and scales
template <int NC>
struct KaStage {
    h8_t k[4][NC][64];                   // [tile][word]
    h8_t v[2][2 * NC][64];               // [pair of tiles][16 columns]
    float ks[64], vs[64];
};

template <int NC, int R, int DT>
__global__ __launch_bounds__(64 * kWaves) void k_kv4_many(KaArgs a)
{
    constexpr int TR = 16 * R * kWaves, KT = 64;
    typedef KaStage<NC> Stage;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    Stage* stage = (Stage*)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g4 = lane >> 4;
    const int h = blockIdx.x % a.H, split = (blockIdx.x / a.H) % a.splits, tile = blockIdx.x / a.H / a.splits;
    int bad = 0;
    KaSeq s;
    int64_t b, row0;
    const bool have = ka_tile<TR, false>(a, tile, s, b, row0, bad);
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
    if (!have) return;
    const int64_t rows = s.n * a.G;

    // keys of the block's rows in stages, dealt to the splits
    int64_t l0, h0, l1, h1;
    ka_span(a, s, row0, l0, h0);
    ka_span(a, s, (row0 + TR < rows ? row0 + TR : rows) - 1, l1, h1);
    const int32_t k_lo = (int32_t)l0 & ~(KT - 1), k_hi = (int32_t)h1, kv = (int32_t)s.kv;
    const int32_t steps = k_hi > k_lo ? (k_hi - k_lo + KT - 1) / KT : 0;
    const int32_t per = (steps + a.splits - 1) / a.splits, it0 = split * per;
    const int32_t n_it = it0 + per < steps ? per : (steps > it0 ? steps - it0 : 0);
    const int32_t key0 = k_lo + it0 * KT;

    // one half of the waves bring a tile of keys each, the other one nibble of a
    // pair of tiles of values and the scales of one tile
    KaTiles<4, 4> tl = {a.table + b * a.table_ld, key0 >> 4, (int32_t)l0 >> 4, (kv + 15) >> 4, 0, -1, 0};
    const bool values = wave >= 4;
    const int own = wave & 3, vn = wave & 1;
    KaWords<NC> wa, wb;
    float sc = 0.f;
    auto fetch = [&](int it) {
        if (it % tl.N == 0) tl.look(a, h, it);
        const int ti = tl.at(it, own);
        const int64_t o = ti >= 0 ? ti : 0;
        if (!values) {
            wa = words<NC>(a.kc + o * (256 * NC) + (c * 4 + g4) * (4 * NC));
            wb = wa;
            sc = a.ks[o * 16 + c];
        } else {
            const int u0 = tl.at(it, own & ~1), u1 = tl.at(it, own | 1);
            const int64_t t0 = u0 >= 0 ? u0 : 0, t1 = u1 >= 0 ? u1 : 0;
            wa = words<NC>(a.vc + t0 * (256 * NC) + (c * 4 + g4) * (4 * NC));
            wb = words<NC>(a.vc + t1 * (256 * NC) + (c * 4 + g4) * (4 * NC));
            sc = a.vs[o * 16 + c];
        }
    };
    auto spread = [&](Stage& d) {
        if (!values) {
#pragma unroll
            for (int w = 0; w < NC; w++) {
                const uint32_t u = wa.w[w], v = u >> 8;
                d.k[own][w][lane] = join8(codes_lo(u), codes_hi(u), codes_lo(v), codes_hi(v));
            }
            if (lane < 16) d.ks[own * 16 + lane] = sc * KaRows<NC, R, DT>::k_down;
        } else {
#pragma unroll
            for (int w = 0; w < NC; w++) {
                const uint32_t a0 = wa.w[w] >> (4 * vn), a1 = wb.w[w] >> (4 * vn), b0 = a0 >> 8, b1 = a1 >> 8;
                d.v[own >> 1][2 * w + vn][lane] = join8(codes_lo(a0), codes_lo(b0), codes_lo(a1), codes_lo(b1));
            }
            if (lane < 16) d.vs[own * 16 + lane] = sc;
        }
    };
    if (n_it > 0) {
        tl.ask(a, 0);
        fetch(0);                        // under way while the queries come
    }
    KaRows<NC, R, DT> x;
    x.load(a, s, row0 + wave * 16 * R, rows, h);
    uint32_t ok_now = 0, ok_next = 0;    // tiles that are there, taken before the next look-up
    if (n_it > 0) {
        ok_next = tl.mask(0);
        spread(stage[0]);
        if (n_it > 1) fetch(1);
    }
    for (int it = 0; it < n_it; it++) {
        __syncthreads();
        ok_now = ok_next;
        if (it + 1 < n_it) {
            ok_next = tl.mask(it + 1);
            spread(stage[(it + 1) & 1]);
            if (it + 2 < n_it) fetch(it + 2);
        }
        const int32_t kb = key0 + it * KT;
        if (kb >= x.any_hi || kb + KT <= x.any_lo) continue;
        const Stage& y = stage[it & 1];
        f4_t st[R][4], ks[4], vs[4];
        bool ok[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            ok[i] = ok_now >> i & 1;
            ks[i] = *(const f4_t*)(y.ks + i * 16 + g4 * 4);
            vs[i] = *(const f4_t*)(y.vs + i * 16 + g4 * 4);
#pragma unroll
            for (int t = 0; t < R; t++) st[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NC; w++) x.score(y.k[i][w][lane], w, i, st);
        }
        h8_t pf[x.NS][R][2];
        x.soften(st, ks, vs, ok, kb, kv, pf);
#pragma unroll
        for (int p = 0; p < 2; p++)
#pragma unroll
            for (int d = 0; d < 2 * NC; d++) x.add(y.v[p][d][lane], d, p, pf);
    }
#pragma unroll
    for (int t = 0; t < R; t++) {
        const float l = sum4(x.l[t]);
        const int r = wave * 16 * R + t * 16 + c;
        if (row0 + r >= rows) continue;
        const KaOut o = ka_row<TR>(a, s, tile, h, split, row0, r, x.m[t], l, g4 == 0);
#pragma unroll
        for (int i = 0; i < 2 * NC; i++) ka_put(a, o, i * 16 + g4 * 4, x.acc[t][i] * (1.f / x.up[t]));
    }
}

// The splits' parts of the few rows: a block a row, whose groups of W / 4 threads take
// every so many splits; the groups are added in their order.  4.6 us at 32 rows of 96
// parts, 5.9 at 2048 of three: a launch and two trips to memory.
template <int TR>
__global__ __launch_bounds__(256) void k_kv4_join(KaArgs a)
{
    __shared__ float fs[kSplitsMax];
    __shared__ f4_t red[256];
    __shared__ float lsum;
    const int r = blockIdx.x % a.join_rows, h = (blockIdx.x / a.join_rows) % a.H, tile = blockIdx.x / a.join_rows / a.H;
    int bad = 0;
    KaSeq s;
    int64_t b, row0;
    if (!ka_tile<TR, true>(a, tile, s, b, row0, bad)) return;
    if (row0 + r >= s.n * a.G) return;
    const int64_t at = (((int64_t)tile * a.H + h) * TR + r) * a.splits;
    const int lw = a.W / 4, groups = 256 / lw, grp = threadIdx.x / lw, d = (threadIdx.x - grp * lw) * 4;
    if (threadIdx.x < 64) {
        float m[kSplitsMax / 64], mr = kNone, lr = 0.f;
#pragma unroll
        for (int i = 0; i < kSplitsMax / 64; i++) {
            const int k = i * 64 + threadIdx.x;
            m[i] = k < a.splits ? a.pm[(at + k) * 2] : kNone;
            mr = fmaxf(mr, m[i]);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mr = fmaxf(mr, __shfl_xor(mr, o, 64));
#pragma unroll
        for (int i = 0; i < kSplitsMax / 64; i++) {
            const int k = i * 64 + threadIdx.x;
            if (k < a.splits) {
                const float f = __builtin_amdgcn_exp2f(m[i] - mr);
                fs[k] = f;
                lr += f * a.pm[(at + k) * 2 + 1];
            }
        }
        lr = wave_sum_f32(lr);
        if (threadIdx.x == 0) {
            lsum = lr;
            if (a.lse) {
                const int64_t tok = s.q0 + (row0 + r) / a.G, head = h * a.G + (row0 + r) % a.G;
                a.lse[tok * a.Hq + head] = ka_lse(a, mr, lr);
            }
        }
    }
    __syncthreads();
    f4_t o = {0.f, 0.f, 0.f, 0.f};
    if (grp < groups) {
#pragma unroll 4
        for (int i = grp; i < a.splits; i += groups) o += fs[i] * *(const f4_t*)(a.po + (at + i) * a.W + d);
    }
    red[threadIdx.x] = o;
    __syncthreads();
    if (grp == 0 && d < a.D) {
        for (int g = 1; g < groups; g++) o += red[g * lw + threadIdx.x];
        const int64_t tok = s.q0 + (row0 + r) / a.G, head = h * a.G + (row0 + r) % a.G;
        ka_store(a, tok * a.o_ld + head * a.o_hs, d, o, ka_inv(lsum));
    }
}

// The same for the rows of a tile of many: a group of W / 4 threads a row, the parts one
// after the other (4000 rows of 8 heads in two parts: a block a row 63 us, so about 13).
template <int TR>
__global__ __launch_bounds__(256) void k_kv4_join_many(KaArgs a)
{
    const int lw = a.W / 4, rpb = 256 / lw, bpt = (TR + rpb - 1) / rpb, grp = threadIdx.x / lw, d = (threadIdx.x - grp * lw) * 4;
    const int h = (blockIdx.x / bpt) % a.H, tile = blockIdx.x / bpt / a.H, r = blockIdx.x % bpt * rpb + grp;
    int bad = 0;
    KaSeq s;
    int64_t b, row0;
    if (!ka_tile<TR, false>(a, tile, s, b, row0, bad)) return;
    if (grp >= rpb || r >= TR || row0 + r >= s.n * a.G) return;
    const int64_t at = (((int64_t)tile * a.H + h) * TR + r) * a.splits;
    float mr = kNone, lr = 0.f;
    for (int i = 0; i < a.splits; i++) mr = fmaxf(mr, a.pm[(at + i) * 2]);
    f4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < a.splits; i++) {
        const float f = __builtin_amdgcn_exp2f(a.pm[(at + i) * 2] - mr);
        lr += f * a.pm[(at + i) * 2 + 1];
        o += f * *(const f4_t*)(a.po + (at + i) * a.W + d);
    }
    const int64_t q = (row0 + r) / a.G, tok = s.q0 + q, head = h * a.G + (row0 + r - q * a.G);
    if (a.lse && d == 0) a.lse[tok * a.Hq + head] = ka_lse(a, mr, lr);
    if (d < a.D) ka_store(a, tok * a.o_ld + head * a.o_hs, d, o, ka_inv(lr));
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// A call's launches: requests of up to 16 R rows by blocks whose waves share
// them, the others in tiles of many_rows.
struct KaPlan {
    int R;                       // tiles of 16 rows of the first kind; 0: none
    int64_t tiles2;              // of the second kind; 0: none
    int R2, many_rows;
    int splits, splits2;
    size_t part, bytes;
};

// what a wave's registers hold
constexpr int ka_many(int nc, int dt) { return dt == ISEG_F32 || nc > 4 ? 1 : 2; }
constexpr int ka_few_most(int nc, int dt) { return dt == ISEG_F32 ? (nc <= 4 ? 2 : 1) : (nc <= 4 ? 4 : 2); }

int64_t ka_max_kv(const iseg_kv4_attention_geom* g)
{
    const int64_t most = g->n_pages > 0 ? g->max_pages * g->page : 0;
    return g->max_kv > 0 && g->max_kv < most ? g->max_kv : most;
}

int64_t ka_max_q(const iseg_kv4_attention_geom* g) { return g->max_q > 0 && g->max_q < g->T ? g->max_q : g->T; }

// Time of n tiles (with all heads) in sp splits, in stages of 64 keys for 256 rows (3.8
// us): a block a CU at a time, each with three stages of beginning and end, the longest
// first.  With one tile of 16 rows a wave a stage is taken as 0.72 of that for 128 rows; it
// is 0.55 where blocks follow one another (3 x 3001 in tiles of 128 1290 us, of 256 1180),
// but whole rounds of blocks count more of them than there are.  The queries of a prompt
// see half of its own keys.  Splits write and read parts.  Without it (256 rows always,
// splits for one round of blocks rounded up): 128 rows behind 131072 keys 199 us, 148 now;
// a prompt of 512 38, 27 now, of 1000 59, 44 now; 100 tokens behind 99900 332 both, 16 x 300
// 93 both (90 in tiles of 128).
double ka_cost(const iseg_kv4_attention_geom* g, int R, int64_t n, int sp, int64_t span)
{
    const double stages = span / 64 + 1, own = g->causal ? (double)(ka_max_q(g) < span ? ka_max_q(g) : span) / 128 : 0.0;
    const double rounds = (double)ceil_div64(n * sp, 256), mean = rounds / sp * (stages - own);
    const double time = (stages / sp > mean ? stages / sp : mean) + 3.0 * rounds;
    const double parts = sp > 1 ? 2.0 + (double)(g->T * g->Hq * sp) * kv4_width(g->D) / 1.5e6 : 0.0;
    return (R == 1 ? 0.72 : 1.0) * time + parts;
}

KaPlan ka_plan(const iseg_kv4_attention_geom* g)
{
    KaPlan p = {};
    const int nc = kv4_width(g->D) / 32;
    const int64_t G = g->Hq / g->H, rows = ka_max_q(g) * G, pairs = g->B * g->H;
    const int most = ka_few_most(nc, g->dtype);
    int64_t span = ka_max_kv(g);
    if (g->window > 0 && g->window + ka_max_q(g) < span) span = g->window + ka_max_q(g);
    if (rows <= 16 * most || g->B > 1) {
        const int64_t r = rows <= 16 * most ? rows : 16 * most;
        p.R = r <= 16 ? 1 : (r <= 32 ? 2 : 4);
        // Few pairs of request and head: as many blocks as are resident, all of one
        // length (1 request of 131072 keys, 8 heads: a call 38 us at 96 splits, 43 at 128).
        // Many: two rounds of blocks, which even out requests of different lengths (64
        // of 820 to 8192 keys: 95 us against 98 in one; 64 x 8192 124 both; heads of 256, 32 x
        // 8192, 140 against 129).
        const int64_t resident = 256 * ka_few_waves(nc, p.R, g->dtype);
        int64_t sp = 8 * pairs <= resident ? resident / pairs : ceil_div64(2 * resident, pairs), longest = ceil_div64(span, 256);
        sp = sp < longest ? sp : longest;
        p.splits = (int)(sp < 1 ? 1 : (sp > kSplitsMax ? kSplitsMax : sp));
    }
    if (rows > 16 * most) {
        // requests of more rows than the first kind's, each with a last tile that may not
        // be full
        const int64_t large = g->T * G / (p.R ? 16 * p.R + 1 : 1), ends = large < g->B ? large : g->B;
        double best = 0.0;
        for (int R = ka_many(nc, g->dtype); R >= 1; R--) {
            const int64_t TR = 16 * kWaves * R, all = (g->T * G - ends) / TR + ends, each = ends * ceil_div64(rows, TR);
            const int64_t tiles = all < each ? all : each;
            for (int sp = 1; sp <= 32 && (sp == 1 || sp * 512 <= span); sp++) {
                const double c = ka_cost(g, R, tiles * g->H, sp, span);
                if (p.tiles2 > 0 && c >= best) continue;
                best = c;
                p.R2 = R;
                p.many_rows = (int)TR;
                p.tiles2 = tiles;
                p.splits2 = sp;
            }
        }
    }
    const int64_t n1 = p.R && p.splits > 1 ? pairs * 16 * p.R * p.splits : 0;
    const int64_t n2 = p.splits2 > 1 ? p.tiles2 * g->H * p.many_rows * p.splits2 : 0;
    const int64_t n = n1 > n2 ? n1 : n2;
    p.part = align256((size_t)n * 8);
    p.bytes = n ? ws_used(p.part + (size_t)n * kv4_width(g->D) * 4) : kNoWs;
    return p;
}

int ka_check(const iseg_kv4_attention_geom* g)
{
    if (!g || !is_float_dtype(g->dtype) || g->causal < 0 || g->causal > 1 || !(g->scale > 0.f && g->scale <= 3.4028234e38f))
        return ISEG_ERR_ARG;
    if (g->T < 0 || g->B < 0 || g->H < 1 || g->Hq < 1 || g->Hq % g->H || g->D < 1 || g->T >= (int64_t)1 << 31 || g->B >= (int64_t)1 << 31 ||
        g->q_ld < 0 || g->q_hs < 0 || g->n_pages < 0 || g->max_pages < 0 || g->table_ld < g->max_pages || g->max_q < 0 ||
        g->max_kv < 0 || g->window < 0 || g->page < 16 || g->page % 16 || !rows_apart(g->T, g->Hq, g->D, g->o_ld, g->o_hs))
        return ISEG_ERR_SHAPE;
    if (g->D % 8 || g->D > 256 || g->page > 8192 || g->Hq > 65536 || !kv4_pages_ok(g->n_pages, g->page) ||
        g->max_pages >= (int64_t)1 << 27 || ka_max_kv(g) >= ((int64_t)1 << 31) - (1 << 16) ||
        g->n_pages * g->H * (g->page / 16) >= (int64_t)1 << 31 || g->window >= (int64_t)1 << 40)
        return ISEG_ERR_UNSUPPORTED;
    if (g->T > 0 && g->B > 0) {
        const KaPlan p = ka_plan(g);
        const int64_t most = (int64_t)1 << 24;               // blocks of 256 threads of a launch, half of 512
        if (g->B * g->H * p.splits >= most || (p.splits > 1 && g->B * g->H * 16 * p.R >= most) ||
            p.tiles2 * g->H * p.splits2 >= most / 2 || (p.splits2 > 1 && p.tiles2 * g->H * p.many_rows >= most))
            return ISEG_ERR_UNSUPPORTED;
    }
    return ISEG_OK;
}

template <int NC, int R, int DT>
int ka_few(KaArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((k_kv4_few<NC, R, DT>), dim3((unsigned)((int64_t)a.B * a.H * a.splits)), dim3(256), 0, s, a);
    const int64_t rows = a.max_q * a.G;
    a.join_rows = (int32_t)(rows < 16 * R ? rows : 16 * R);
    if (a.splits > 1)
        hipLaunchKernelGGL((k_kv4_join<16 * R>), dim3((unsigned)((int64_t)a.B * a.H * a.join_rows)), dim3(256), 0, s, a);
    return launch_ok();
}

template <int NC, int R, int DT>
int ka_many_rows(const KaArgs& a, const KaPlan& p, hipStream_t s)
{
    constexpr size_t lds = 2 * sizeof(KaStage<NC>);
    constexpr int TR = 16 * kWaves * R, rpb = 256 / (NC * 8);
    if (!lds_limit((const void*)&k_kv4_many<NC, R, DT>, lds)) return ISEG_ERR_DEVICE;
    hipLaunchKernelGGL((k_kv4_many<NC, R, DT>), dim3((unsigned)(p.tiles2 * a.H * a.splits)), dim3(64 * kWaves), lds, s, a);
    if (a.splits > 1)
        hipLaunchKernelGGL((k_kv4_join_many<TR>), dim3((unsigned)(p.tiles2 * a.H * ((TR + rpb - 1) / rpb))), dim3(256), 0, s, a);
    return launch_ok();
}

template <int NC, int DT>
int ka_run(KaArgs a, const KaPlan& p, hipStream_t s)
{
    constexpr int most = ka_few_most(NC, DT);
    int rc = ISEG_OK;
    if (p.R) {
        a.rows_min = 0;
        a.rows_max = 16 * p.R;
        a.splits = p.splits;
        if (p.R == 1) rc = ka_few<NC, 1, DT>(a, s);
        if constexpr (most >= 2)
            if (p.R == 2) rc = ka_few<NC, 2, DT>(a, s);
        if constexpr (most >= 4)
            if (p.R == 4) rc = ka_few<NC, 4, DT>(a, s);
    }
    if (rc == ISEG_OK && p.tiles2 > 0) {
        a.rows_min = p.R ? 16 * p.R : 0;
        a.rows_max = 0x7fffffff;
        a.splits = p.splits2;
        constexpr int R = ka_many(NC, DT);
        rc = R == 1 || p.R2 == 1 ? ka_many_rows<NC, 1, DT>(a, p, s) : ka_many_rows<NC, R, DT>(a, p, s);
    }
    return rc;
}

template <int DT>
int ka_widths(const KaArgs& a, const KaPlan& p, hipStream_t s)
{
    switch (a.W / 32) {
    case 1: return ka_run<1, DT>(a, p, s);
    case 2: return ka_run<2, DT>(a, p, s);
    case 3: return ka_run<3, DT>(a, p, s);
    case 4: return ka_run<4, DT>(a, p, s);
    case 6: return ka_run<6, DT>(a, p, s);
    default: return ka_run<8, DT>(a, p, s);
    }
}

}  // namespace

extern "C" size_t iseg_kv4_attention_ws(const iseg_kv4_attention_geom* g)
{
    if (ka_check(g) != ISEG_OK) return 0;
    return g->T > 0 && g->B > 0 ? ka_plan(g).bytes : kNoWs;
}

extern "C" int iseg_kv4_attention(const void* q, const uint8_t* k_codes, const float* k_scale, const uint8_t* v_codes,
                                  const float* v_scale, const int32_t* table, const int32_t* q_start,
                                  const int32_t* kv_len, const iseg_kv4_attention_geom* g, void* out, float* lse,
                                  void* ws, size_t ws_bytes, int32_t* dev_status, hipStream_t stream)
{
    const int rc = ka_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->T == 0 || g->B == 0) return ISEG_OK;
    if (!q || !out || !q_start || !kv_len ||
        (ka_max_kv(g) > 0 && (!k_codes || !k_scale || !v_codes || !v_scale || !table)))
        return ISEG_ERR_ARG;
    if (((uintptr_t)k_codes | (uintptr_t)v_codes | (uintptr_t)k_scale | (uintptr_t)v_scale) & 15) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_kv4_attention_ws(g)) return ISEG_ERR_WORKSPACE;
    const KaPlan p = ka_plan(g);
    KaArgs a = {};
    a.q = q; a.kc = k_codes; a.vc = v_codes; a.ks = k_scale; a.vs = v_scale; a.table = table; a.q_start = q_start;
    a.kv_len = kv_len; a.out = out; a.lse = lse;
    a.pm = (float*)ws;
    a.po = (float*)((char*)ws + p.part);
    a.T = g->T; a.q_ld = g->q_ld; a.q_hs = g->q_hs; a.o_ld = g->o_ld; a.o_hs = g->o_hs; a.table_ld = g->table_ld;
    a.n_pages = g->n_pages; a.max_pages = g->max_pages; a.max_q = ka_max_q(g); a.max_kv = ka_max_kv(g);
    a.window = g->window; a.B = (int32_t)g->B; a.Hq = (int32_t)g->Hq; a.H = (int32_t)g->H; a.G = (int32_t)(g->Hq / g->H);
    a.D = (int32_t)g->D; a.W = kv4_width(g->D); a.p16 = g->page / 16;
    a.p16_inv = (((uint64_t)1 << 36) + a.p16 - 1) / a.p16;
    a.dtype = g->dtype; a.causal = g->causal; a.status = dev_status;
    const double scale = (double)g->scale * 1.442695040888963407;
    a.scale = (float)scale;
    a.scale_left = scale / (double)a.scale;
    return g->dtype == ISEG_F32 ? ka_widths<ISEG_F32>(a, p, stream)
                                : g->dtype == ISEG_F16 ? ka_widths<ISEG_F16>(a, p, stream) : ka_widths<ISEG_BF16>(a, p, stream);
}
