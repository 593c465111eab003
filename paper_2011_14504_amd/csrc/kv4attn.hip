// kv4attn.hip -- attention over the paged 4-bit cache (iseg_kv4_attention).
//
// Rows are the queries of one key head: row r of a request is query r / G, head
// r % G of the G query heads that share it.  A wave takes 16 R rows and steps
// over 32 keys at a time:
//   S^T = K Q^T   on 16x16x32 float16 MFMAs, the codes as A: their scales are a
//                 factor per row of S^T;
//   p = 2^(s - m) with the running maximum m of a row (moved only when a score
//                 passes it by 8: float16 has the room), l += p;
//   O^T += V^T P^T, P in the registers that S^T left it in.  V's scale goes into
//                 p, in float16 relative to the largest scale seen (a power of
//                 two, also moved only when it must be).
// Codes become float16 by placing them in the mantissa of 1024 (9 instructions
// for 8 codes); the layout of the cache makes a lane's operands whole words.
#include "kv4.h"

namespace {

typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef float f4_t __attribute__((ext_vector_type(4)));

constexpr float kNone = -3.0e38f;        // maximum of a row that has seen no key
constexpr float kRoom = 8.f;             // scores may pass the running maximum by 2^8

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
    int32_t rows_min, rows_max;          // rows of the requests that this launch takes: (min, max]
    float scale;                         // times log2 e
    int32_t* status;
};

// eight float16 of a word of K: codes n + 8 in nibbles 0 4 1 5 (and 2 6 3 7 above)
__device__ __forceinline__ h2_t codes_lo(uint32_t w)
{
    const h2_t k = {(_Float16)1032.f, (_Float16)1032.f};
    return __builtin_bit_cast(h2_t, (w & 0x000f000fu) | 0x64006400u) - k;
}

__device__ __forceinline__ h2_t codes_hi(uint32_t w)
{
    const h2_t s = {(_Float16)0.0625f, (_Float16)0.0625f}, k = {(_Float16)-72.f, (_Float16)-72.f};
    return __builtin_elementwise_fma(__builtin_bit_cast(h2_t, (w & 0x00f000f0u) | 0x64006400u), s, k);
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
    if (s.n > a.max_q) bad = 1;
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
            const int64_t end = base + __shfl(sum, at, 64);
            b = b0 + at;
            int ignored = 0;
            s = ka_seq(a, b, ignored);
            row0 = (end - 1 - tile) * TR;
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

template <int NC>
struct KaKeys {                          // 32 keys of one head: a lane's words and scales
    uint32_t k[2][NC], v[2][NC];
    f4_t ks[2], vs[2];
    bool ok[2];
};

template <int NC>
__device__ __forceinline__ void words(const uint8_t* p, uint32_t* w)
{
    __builtin_memcpy(w, __builtin_assume_aligned(p, NC % 4 == 0 ? 16 : NC % 2 == 0 ? 8 : 4), NC * 4);
}

// NC: words of a row's quarter (W / 32).  R: tiles of 16 rows a wave holds.
// SHARED: the four waves hold the same rows and deal the keys among themselves;
// otherwise each has rows of its own and sees all keys.  WIDE: q and p as two
// float16 terms (float32 tensors).
template <int NC, int R, bool SHARED, bool WIDE>
__global__ __launch_bounds__(256) void k_kv4_attention(KaArgs a)
{
    constexpr int W = NC * 32, TR = SHARED ? 16 * R : 64 * R, NS = WIDE ? 2 : 1;
    __shared__ float so[SHARED ? 4 * 16 * (W + 4) : 1];
    __shared__ float sm[4][16], sl[4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g4 = lane >> 4;
    const int h = blockIdx.x % a.H, split = (blockIdx.x / a.H) % a.splits, tile = blockIdx.x / a.H / a.splits;
    int bad = 0;
    KaSeq s;
    int64_t b, row0;
    const bool have = ka_tile<TR, SHARED>(a, tile, s, b, row0, bad);
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
    if (!have) return;
    const int64_t rows = s.n * a.G;
    if (!SHARED) row0 += wave * 16 * R;

    // the wave's rows: keys they see, and their queries as B operands
    int64_t lo[R], hi[R];
    h8_t qf[NS][R][NC];
    float cf[R];
#pragma unroll
    for (int t = 0; t < R; t++) {
        const int64_t r = row0 + t * 16 + c;
        const bool in = r < rows;
        lo[t] = hi[t] = 0;
        if (in) ka_span(a, s, r, lo[t], hi[t]);
        const int64_t at = in ? (s.q0 + r / a.G) * a.q_ld + (h * a.G + r % a.G) * a.q_hs : 0;
        float f[NC][8];
        float big = 0.f;
#pragma unroll
        for (int w = 0; w < NC; w++) {
            const int d = g4 * 8 * NC + w * 8;
#pragma unroll
            for (int i = 0; i < 8; i++) f[w][i] = 0.f;
            if (in && d < a.D) {
                if (WIDE) {
                    float x[8];
                    __builtin_memcpy(x, (const float*)a.q + at + d, 32);
#pragma unroll
                    for (int i = 0; i < 8; i++) f[w][i] = x[i];
                } else if (a.dtype == ISEG_F16) {
                    _Float16 x[8];
                    __builtin_memcpy(x, (const _Float16*)a.q + at + d, 16);
#pragma unroll
                    for (int i = 0; i < 8; i++) f[w][i] = (float)x[i];
                } else {
                    __bf16 x[8];
                    __builtin_memcpy(x, (const __bf16*)a.q + at + d, 16);
#pragma unroll
                    for (int i = 0; i < 8; i++) f[w][i] = (float)x[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; i++) big = fmaxf(big, fabsf(f[w][i]));
        }
        // float16 reaches no further than 65504 and 2^-24: rows of the other
        // types are brought below 1 by a power of two first
        int e = 0;
        if (WIDE || a.dtype != ISEG_F16) {
            big = max4(big);
            if (big > 0.f && big <= 3.4028234e38f) (void)frexpf(big, &e);
            e = e < -100 ? -100 : e;
        }
        cf[t] = fmaxf(ldexpf(a.scale, e), 1.17549435e-38f);      // never 0: a masked score is -infinity times this
#pragma unroll
        for (int w = 0; w < NC; w++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = ldexpf(f[w][i], -e);
                qf[0][t][w][i] = (_Float16)x;
                if constexpr (WIDE) qf[NS - 1][t][w][i] = (_Float16)(x - (float)(_Float16)x);
            }
    }

    // keys of the block (SHARED) or the wave: whole steps, dealt to the splits
    const int64_t r_end = row0 + 16 * R < rows ? row0 + 16 * R : rows;
    int64_t lo_first = 0, hi_first = 0, lo_last = 0, hi_last = 0;
    if (row0 < rows) {
        ka_span(a, s, row0, lo_first, hi_first);
        ka_span(a, s, r_end - 1, lo_last, hi_last);
    }
    constexpr int STEP = SHARED ? 128 : 32;
    const int64_t k_lo = lo_first & ~(int64_t)31;
    const int64_t steps = hi_last > k_lo ? (hi_last - k_lo + STEP - 1) / STEP : 0;
    const int64_t per = (steps + a.splits - 1) / a.splits;
    const int64_t it0 = split * per;
    const int n_it = (int)(it0 + per < steps ? per : (steps > it0 ? steps - it0 : 0));
    const int32_t key0 = (int32_t)(k_lo + it0 * STEP + (SHARED ? wave * 32 : 0));
    const int32_t kv = (int32_t)s.kv;
    const int32_t full_lo = (int32_t)lo_last, full_hi = (int32_t)hi_first;

    // tiles of 16 tokens for 32 steps at a time, a lane each: -1 past the keys or
    // with a page id out of range
    const int32_t* row_table = a.table + b * a.table_ld;
    int tidx = -1;
    auto fetch_tiles = [&](int it) {
        const int32_t t16 = (key0 >> 4) + (it + (lane >> 1)) * (STEP / 16) + (lane & 1);
        const int32_t col = (int32_t)(((uint64_t)(uint32_t)t16 * a.p16_inv) >> 36);
        tidx = -1;
        if (t16 < (kv + 15) >> 4) {
            const int32_t pg = row_table[col];
            if (pg >= 0 && pg < a.n_pages) tidx = (pg * a.H + h) * a.p16 + (t16 - col * a.p16);
            else set_status(a.status, ISEG_DEV_RANGE);
        }
    };
    KaKeys<NC> nx;
    auto fetch = [&](int it) {
        if ((it & 31) == 0) fetch_tiles(it);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int ti = __builtin_amdgcn_readlane(tidx, (it & 31) * 2 + i);
            nx.ok[i] = ti >= 0;
            const int64_t at = ti >= 0 ? ti : 0;
            words<NC>(a.kc + at * (256 * NC) + (c * 4 + g4) * (4 * NC), nx.k[i]);
            words<NC>(a.vc + at * (256 * NC) + (c * 4 + g4) * (4 * NC), nx.v[i]);
            nx.ks[i] = *(const f4_t*)(a.ks + at * 16 + g4 * 4);
            nx.vs[i] = *(const f4_t*)(a.vs + at * 16 + g4 * 4);
        }
    };

    f4_t acc[R][2 * NC];
    float m[R], l[R];
#pragma unroll
    for (int t = 0; t < R; t++) {
        m[t] = kNone;
        l[t] = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * NC; i++) acc[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
    }
    float v_inv = 1.f, v_top = 0.f;      // V's scales times v_inv are below 2^7; up to v_top nothing moves

    if (n_it > 0) fetch(0);
    for (int it = 0; it < n_it; it++) {
        const KaKeys<NC> x = nx;
        if (it + 1 < n_it) fetch(it + 1);
        const int32_t kb = key0 + it * STEP;
        if (SHARED && kb >= (int32_t)hi_last) break;

        f4_t st[R][2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
#pragma unroll
            for (int t = 0; t < R; t++) st[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NC; w++) {
                const uint32_t lo8 = x.k[i][w], hi8 = lo8 >> 8;
                const h8_t kf = join8(codes_lo(lo8), codes_hi(lo8), codes_lo(hi8), codes_hi(hi8));
#pragma unroll
                for (int t = 0; t < R; t++)
#pragma unroll
                    for (int n = 0; n < NS; n++)
                        st[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[n][t][w], st[t][i], 0, 0, 0);
            }
        }

        // V's scales; those of no key count as 0
        f4_t vs[2] = {x.vs[0], x.vs[1]};
        const bool full = x.ok[0] && x.ok[1] && kb >= full_lo && kb + 32 <= full_hi;
        if (!full) {
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int r = 0; r < 4; r++)
                    if (!(x.ok[i] && kb + 16 * i + 4 * g4 + r < kv)) vs[i][r] = 0.f;
        }
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int r = 0; r < 4; r++) top = fmaxf(top, vs[i][r]);
        if (__any(top > v_top)) {
            top = fmaxf(v_top, fminf(max4(top), 3.4028234e38f));
            int e;
            (void)frexpf(top, &e);                               // top in [2^(e-1), 2^e)
            e = e < -100 ? -100 : e;
            const float inv = ldexpf(1.f, 7 - e), f = inv / v_inv;
            v_top = ldexpf(1.f, e);
            v_inv = inv;
#pragma unroll
            for (int t = 0; t < R; t++)
#pragma unroll
                for (int i = 0; i < 2 * NC; i++) acc[t][i] *= f;
        }
#pragma unroll
        for (int i = 0; i < 2; i++) vs[i] *= v_inv;

        float mx[R];
        bool move = false;
#pragma unroll
        for (int t = 0; t < R; t++) {
            mx[t] = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    float v = st[t][i][r] * x.ks[i][r];
                    if (!full) {
                        const int32_t j = kb + 16 * i + 4 * g4 + r;
                        if (!(x.ok[i] && j >= (int32_t)lo[t] && j < (int32_t)hi[t])) v = -__builtin_inff();
                    }
                    st[t][i][r] = v;
                    mx[t] = fmaxf(mx[t], v);
                }
            move = move || mx[t] * cf[t] > m[t] + kRoom;
        }
        if (__any(move)) {
#pragma unroll
            for (int t = 0; t < R; t++) {
                const float mn = fmaxf(m[t], max4(mx[t]) * cf[t]);
                const float al = __builtin_amdgcn_exp2f(m[t] - mn);
                m[t] = mn;
                l[t] *= al;
#pragma unroll
                for (int i = 0; i < 2 * NC; i++) acc[t][i] *= al;
            }
        }
        h8_t pf[NS][R];
#pragma unroll
        for (int t = 0; t < R; t++) {
            float p[2][4];
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float v = __builtin_amdgcn_exp2f(fmaf(st[t][i][r], cf[t], -m[t]));
                    l[t] += v;
                    p[i][r] = v * vs[i][r];
                    if (!full && st[t][i][r] == -__builtin_inff()) p[i][r] = 0.f;      // a masked key's scale may be anything
                }
            // V's words hold tokens 0 2 and 1 3 as pairs
#pragma unroll
            for (int i = 0; i < 2; i++) {
                constexpr int order[4] = {0, 2, 1, 3};
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float v = p[i][order[r]];
                    pf[0][t][4 * i + r] = (_Float16)v;
                    if constexpr (WIDE) pf[NS - 1][t][4 * i + r] = (_Float16)(v - (float)(_Float16)v);
                }
            }
        }
#pragma unroll
        for (int w = 0; w < NC; w++) {
            const uint32_t a0 = x.v[0][w], a1 = x.v[1][w], b0 = a0 >> 8, b1 = a1 >> 8;
            const h8_t vl = join8(codes_lo(a0), codes_lo(b0), codes_lo(a1), codes_lo(b1));
            const h8_t vh = join8(codes_hi(a0), codes_hi(b0), codes_hi(a1), codes_hi(b1));
#pragma unroll
            for (int t = 0; t < R; t++)
#pragma unroll
                for (int n = 0; n < NS; n++) {
                    acc[t][2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, pf[n][t], acc[t][2 * w], 0, 0, 0);
                    acc[t][2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, pf[n][t], acc[t][2 * w + 1], 0, 0, 0);
                }
        }
    }

    // rows out: the whole, or this split's part
    const float v_out = 1.f / v_inv;
    auto put = [&](int64_t r, int d, f4_t o, float mr, float lr) {     // four elements of row r from d on
        if (a.splits > 1) {
            const int64_t at = (((int64_t)tile * a.H + h) * TR + r) * a.splits + split;
            *(f4_t*)(a.po + at * W + d) = o;
            if (d == 0) { a.pm[at * 2] = mr; a.pm[at * 2 + 1] = lr; }
            return;
        }
        const int64_t rr = SHARED ? r : row0 - wave * 16 * R + r;
        const int64_t tok = s.q0 + rr / a.G, head = h * a.G + rr % a.G;
        const float inv = lr > 0.f ? 1.f / lr : (lr == lr ? 0.f : lr);
        if (d < a.D) {
            if (WIDE) {
                float x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
                __builtin_memcpy((float*)a.out + tok * a.o_ld + head * a.o_hs + d, x, 16);
            } else if (a.dtype == ISEG_F16) {
                _Float16 x[4] = {(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
                __builtin_memcpy((_Float16*)a.out + tok * a.o_ld + head * a.o_hs + d, x, 8);
            } else {
                __bf16 x[4] = {(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
                __builtin_memcpy((__bf16*)a.out + tok * a.o_ld + head * a.o_hs + d, x, 8);
            }
        }
        if (d == 0 && a.lse)
            a.lse[tok * a.Hq + head] = lr > 0.f || lr != lr ? (mr + __builtin_amdgcn_logf(lr)) * 0.69314718f : -__builtin_inff();
    };
#pragma unroll
    for (int t = 0; t < R; t++) l[t] = sum4(l[t]);
    if constexpr (!SHARED) {
#pragma unroll
        for (int t = 0; t < R; t++) {
            if (row0 + t * 16 + c >= rows) continue;
#pragma unroll
            for (int i = 0; i < 2 * NC; i++)
                put(wave * 16 * R + t * 16 + c, i * 16 + g4 * 4, acc[t][i] * v_out, m[t], l[t]);
        }
    } else {
        for (int t = 0; t < R; t++) {
            if (t * 16 >= rows) break;
            __syncthreads();
            float* mine = so + (wave * 16 + c) * (W + 4) + g4 * 4;
#pragma unroll
            for (int u = 0; u < R; u++)
                if (u == t) {
#pragma unroll
                    for (int i = 0; i < 2 * NC; i++) *(f4_t*)(mine + i * 16) = acc[u][i] * v_out;
                    if (g4 == 0) { sm[wave][c] = m[u]; sl[wave][c] = l[u]; }
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
                put(t * 16 + r, d, o, mr, lr);
            }
        }
    }
}

// The splits' parts of a row, in their order: a block a row.
template <int TR, bool SHARED>
__global__ __launch_bounds__(64) void k_kv4_join(KaArgs a)
{
    const int r = blockIdx.x % TR, h = (blockIdx.x / TR) % a.H, tile = blockIdx.x / TR / a.H;
    int bad = 0;
    KaSeq s;
    int64_t b, row0;
    if (!ka_tile<TR, SHARED>(a, tile, s, b, row0, bad)) return;
    if (row0 + r >= s.n * a.G) return;
    const int64_t at = (((int64_t)tile * a.H + h) * TR + r) * a.splits;
    float mr = kNone;
    for (int i = threadIdx.x; i < a.splits; i += 64) mr = fmaxf(mr, a.pm[(at + i) * 2]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mr = fmaxf(mr, __shfl_xor(mr, o, 64));
    float lr = 0.f;
    f4_t o = {0.f, 0.f, 0.f, 0.f};
    const int d = threadIdx.x * 4;
    for (int i = 0; i < a.splits; i++) {
        const float f = __builtin_amdgcn_exp2f(a.pm[(at + i) * 2] - mr);
        lr += f * a.pm[(at + i) * 2 + 1];
        if (d < a.W) o += f * *(const f4_t*)(a.po + (at + i) * a.W + d);
    }
    const int64_t tok = s.q0 + (row0 + r) / a.G, head = h * a.G + (row0 + r) % a.G;
    const float inv = lr > 0.f ? 1.f / lr : (lr == lr ? 0.f : lr);
    if (d < a.D) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t p = tok * a.o_ld + head * a.o_hs + d + i;
            if (a.dtype == ISEG_F32) ((float*)a.out)[p] = o[i] * inv;
            else if (a.dtype == ISEG_F16) ((_Float16*)a.out)[p] = (_Float16)(o[i] * inv);
            else ((__bf16*)a.out)[p] = (__bf16)(o[i] * inv);
        }
    }
    if (threadIdx.x == 0 && a.lse)
        a.lse[tok * a.Hq + head] = lr > 0.f || lr != lr ? (mr + __builtin_amdgcn_logf(lr)) * 0.69314718f : -__builtin_inff();
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// A call's launches: requests of up to 16 R rows by blocks whose waves share
// them, the others in tiles of 64 or 128 rows.
struct KaPlan {
    int R;                       // tiles of 16 rows of the first kind; 0: none
    int R2;                      // rows of the second kind's tiles / 64; 0: none
    int64_t tiles2;
    int splits, splits2;
    size_t part, bytes;
};

bool ka_wide(const iseg_kv4_attention_geom* g) { return g->dtype == ISEG_F32; }

int64_t ka_max_kv(const iseg_kv4_attention_geom* g)
{
    const int64_t most = g->n_pages > 0 ? g->max_pages * g->page : 0;
    return g->max_kv > 0 && g->max_kv < most ? g->max_kv : most;
}

int64_t ka_max_q(const iseg_kv4_attention_geom* g) { return g->max_q > 0 && g->max_q < g->T ? g->max_q : g->T; }

KaPlan ka_plan(const iseg_kv4_attention_geom* g)
{
    KaPlan p = {};
    const int nc = kv4_width(g->D) / 32;
    const int64_t G = g->Hq / g->H, rows = ka_max_q(g) * G, pairs = g->B * g->H;
    const int most = ka_wide(g) ? (nc <= 4 ? 2 : 1) : (nc <= 4 ? 4 : 2);     // registers
    int64_t span = ka_max_kv(g);
    if (g->window > 0 && g->window + ka_max_q(g) < span) span = g->window + ka_max_q(g);
    if (rows <= 16 * most || g->B > 1) {
        const int64_t r = rows <= 16 * most ? rows : 16 * most;
        p.R = r <= 16 ? 1 : (r <= 32 ? 2 : 4);
        int64_t sp = ceil_div64(1024, pairs), longest = ceil_div64(span, 256);
        sp = sp < longest ? sp : longest;
        p.splits = (int)(sp < 1 ? 1 : (sp > 128 ? 128 : sp));
    }
    if (rows > 16 * most) {
        p.R2 = ka_wide(g) || nc > 4 ? 1 : 2;
        p.tiles2 = ceil_div64(g->T * G, 64 * p.R2) + g->B;
        int64_t sp = ceil_div64(512, p.tiles2 * g->H), longest = ceil_div64(span, 512);
        sp = sp < longest ? sp : longest;
        p.splits2 = (int)(sp < 1 ? 1 : (sp > 32 ? 32 : sp));
    }
    const int64_t n1 = p.R && p.splits > 1 ? pairs * 16 * p.R * p.splits : 0;
    const int64_t n2 = p.R2 && p.splits2 > 1 ? p.tiles2 * g->H * 64 * p.R2 * p.splits2 : 0;
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
        const int64_t most = (int64_t)1 << 24;               // blocks of 256 threads of a launch
        if (g->B * g->H * p.splits >= most || (p.splits > 1 && g->B * g->H * 16 * p.R >= 4 * most) ||
            (p.R2 && (p.tiles2 * g->H * p.splits2 >= most || (p.splits2 > 1 && p.tiles2 * g->H * 64 * p.R2 >= 4 * most))))
            return ISEG_ERR_UNSUPPORTED;
    }
    return ISEG_OK;
}

template <int NC, int R, bool SHARED, bool WIDE>
int ka_launch(const KaArgs& a, int64_t tiles, hipStream_t s)
{
    constexpr int TR = SHARED ? 16 * R : 64 * R;
    hipLaunchKernelGGL((k_kv4_attention<NC, R, SHARED, WIDE>), dim3((unsigned)(tiles * a.H * a.splits)), dim3(256), 0, s, a);
    if (a.splits > 1)
        hipLaunchKernelGGL((k_kv4_join<TR, SHARED>), dim3((unsigned)(tiles * a.H * TR)), dim3(64), 0, s, a);
    return launch_ok();
}

template <int NC, bool WIDE>
int ka_run(KaArgs a, const KaPlan& p, hipStream_t s)
{
    constexpr int most = WIDE ? (NC <= 4 ? 2 : 1) : (NC <= 4 ? 4 : 2);
    int rc = ISEG_OK;
    if (p.R) {
        a.rows_min = 0;
        a.rows_max = 16 * p.R;
        a.splits = p.splits;
        if (p.R == 1) rc = ka_launch<NC, 1, true, WIDE>(a, a.B, s);
        if constexpr (most >= 2)
            if (p.R == 2) rc = ka_launch<NC, 2, true, WIDE>(a, a.B, s);
        if constexpr (most >= 4)
            if (p.R == 4) rc = ka_launch<NC, 4, true, WIDE>(a, a.B, s);
    }
    if (rc == ISEG_OK && p.R2) {
        constexpr int R2 = WIDE || NC > 4 ? 1 : 2;
        a.rows_min = p.R ? 16 * p.R : 0;
        a.rows_max = 0x7fffffff;
        a.splits = p.splits2;
        rc = ka_launch<NC, R2, false, WIDE>(a, p.tiles2, s);
    }
    return rc;
}

template <bool WIDE>
int ka_widths(const KaArgs& a, const KaPlan& p, hipStream_t s)
{
    switch (a.W / 32) {
    case 1: return ka_run<1, WIDE>(a, p, s);
    case 2: return ka_run<2, WIDE>(a, p, s);
    case 3: return ka_run<3, WIDE>(a, p, s);
    case 4: return ka_run<4, WIDE>(a, p, s);
    case 6: return ka_run<6, WIDE>(a, p, s);
    default: return ka_run<8, WIDE>(a, p, s);
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
    a.dtype = g->dtype; a.causal = g->causal; a.scale = g->scale * 1.44269504f; a.status = dev_status;
    return ka_wide(g) ? ka_widths<true>(a, p, stream) : ka_widths<false>(a, p, stream);
}
