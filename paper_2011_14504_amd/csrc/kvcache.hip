// kvcache.hip -- the paged 4-bit cache: writing and reading tokens (iseg_kv4_write,
// iseg_kv4_read), and the step's pages, slots and positions (iseg_page_map).
#include "coder.h"
#include "kv4.h"

namespace {

// ---------------------------------------------------------------------------
// tokens into the cache and back
// ---------------------------------------------------------------------------
struct KvArgs {
    const void *k, *v, *slots;
    void *ko, *vo;
    uint8_t *kc, *vc;
    float *ks, *vs;
    int64_t T, rows;                 // rows: heads of four tokens, or of one
    int64_t k_ld, k_hs, v_ld, v_hs;
    int64_t n_slots;
    int32_t H, D, W, page, slot64, mode, four;
    int32_t* status;
};

// where a token lies: rows of pages, heads and tokens, counted in tokens
struct KvPlace {
    int64_t row;                     // (page id * H + head) * page + place in the page
    int64_t tile;                    // first byte of its tile of 16 tokens in v
    int t;                           // token of the tile
};

__device__ __forceinline__ KvPlace kv_place(const KvArgs& a, int64_t slot, int h)
{
    const uint32_t s = (uint32_t)slot, pg = s / (uint32_t)a.page, in = s - pg * (uint32_t)a.page;
    KvPlace p;
    p.row = ((int64_t)pg * a.H + h) * a.page + in;
    p.tile = (p.row - (in & 15)) * (a.W / 2);
    p.t = (int)(in & 15);
    return p;
}

__device__ __forceinline__ int64_t kv_slot(const KvArgs& a, int64_t t)
{
    return a.slot64 ? ((const int64_t*)a.slots)[t] : ((const int32_t*)a.slots)[t];
}

// eight elements of a row, as words: halves apart, a wave would wait for them one by one
template <typename T>
struct Kv8 {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(w, p, sizeof(w)); }
    __device__ __forceinline__ void load(const T* p, int n)                  // n of them, then zeros
    {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint32_t v = 0;
            if (i < n) __builtin_memcpy(&v, p + i, sizeof(T));
            if (sizeof(T) == 4) w[i % (2 * sizeof(T))] = v;
            else if (i & 1) w[i / 2] |= v << 16;
            else w[i / 2] = v;
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        else return (float)__builtin_bit_cast(T, (uint16_t)(w[i / 2] >> (i & 1) * 16));
    }
};

// the largest magnitude of eight as its type's own bits: 16-bit types two at a time
template <typename T>
__device__ __forceinline__ uint32_t kv_big(const Kv8<T>& r)
{
    if constexpr (sizeof(T) == 4) {
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t b = r.w[i] & 0x7fffffffu;
            big = b > big ? b : big;
        }
        return big;
    } else {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 m = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r.w[i] & 0x7fff7fffu));
        return m.x > m.y ? m.x : m.y;
    }
}

// a magnitude's bits as those of the float32 that it is
template <typename T>
__device__ __forceinline__ uint32_t kv_bits(uint32_t big)
{
    if constexpr (sizeof(T) == 4) return big;
    else return bits_of((float)__builtin_bit_cast(T, (uint16_t)big));
}

// the maximum over LPR lanes, in all of them
template <int LPR>
__device__ __forceinline__ uint32_t kv_max(uint32_t v)
{
    v = dpp_max_step<0xb1>(v);                         // the other of two, of two pairs,
    v = dpp_max_step<0x4e>(v);
    if (LPR >= 8) v = dpp_max_step<0x141>(v);          // of eight turned round, of sixteen
    if (LPR >= 16) v = dpp_max_step<0x140>(v);
    if (LPR >= 32) {
        const uint32_t t = (uint32_t)__shfl_xor((int)v, 16, 64);
        v = t > v ? t : v;
    }
    return v;
}

// lane q's value in its four lanes
template <int Q>
__device__ __forceinline__ uint32_t kv_from(uint32_t v, int q)
{
    if (Q == 1) return v;
    switch (q) {
    case 0: return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x00, 0xf, 0xf, false);
    case 1: return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x55, 0xf, 0xf, false);
    case 2: return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0xaa, 0xf, 0xf, false);
    default: return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0xff, 0xf, 0xf, false);
    }
}

// Scale of a largest magnitude given as float32 bits: scale_of (coder.h) with 4
// bits, in float32.  A float32 quotient rounded once is the float64 one rounded to
// float32 (24 bits twice and two more fit in 53).
__device__ __forceinline__ float kv_scale(uint32_t big, int mode)
{
    if (big >= 0x7f800000u) return __builtin_nanf("");
    const float t = __builtin_bit_cast(float, big);
    float s = t / 7.f;
    if (mode == ISEG_SCALE_POW2) {
        int e;
        (void)frexpf(t, &e);                           // t = f 2^e with f in [1/2, 1): 2^e is the power above t
        s = big ? ldexpf(1.f, e - 3) : 0.f;
    }
    return s < kKvScaleMin ? kKvScaleMin : s;
}

// The codes clamp(floor(v / s + 1/2), +-7) + 8 of eight elements in bits 19 to 22 of
// x.  With v / s + 24.5 in [16, 32) the mantissa's first four bits are the code and
// its other 19 the distance from the half-step below it.  The float32 sum is within
// half a unit of 2^-19 of its terms' (the fma's one rounding) and 8 2^-24 of v / s
// (1 / s rounded), together less than one: the floor can differ only where those 19
// bits are zero, and there only from below, when v - (n - 1/2) s < 0.  That
// remainder's sign is exact however its fma rounds.  s is in [2^-60, 2^126): its
// reciprocal is normal, and v / s is at most 8, which only a power of two passes 7.5
// with; the clamp leaves the outermost codes' middle.
__device__ __forceinline__ void kv_codes(const float* f, float s, float inv, uint32_t* x)
{
    uint32_t near = ~0u;
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        t[e] = __builtin_amdgcn_fmed3f(fmaf(f[e], inv, 24.5f), 17.5f, 31.5f);
        x[e] = __builtin_bit_cast(uint32_t, t[e]);
        const uint32_t frac = x[e] << 13;
        near = frac < near ? frac : near;
    }
    if (near == 0) {
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] -= (uint32_t)((x[e] << 13 == 0) & (fmaf(24.5f - t[e], s, f[e]) < 0.f)) << 19;
    }
}

// byte 2 of four words
__device__ __forceinline__ uint32_t kv_gather(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0602), __builtin_amdgcn_perm(b, a, 0x0c0c0602), 0x05040100);
}

// codes in bits 3 to 6 of each byte to low and high halves
__device__ __forceinline__ uint32_t kv_halves(uint32_t lo, uint32_t hi) { return (lo >> 3 & 0x0f0f0f0fu) | (hi << 1 & 0xf0f0f0f0u); }

// LPR lanes a row, eight columns (a word of codes) a lane, four tokens of a head
// at a time (Q = 4); blockIdx.y: keys or values.  What is the same for a row (its
// place, its scale and that one's reciprocal) each of four lanes has for one of the
// four tokens.  A byte of v holds columns 16 apart, which lie two lanes apart: each
// pair of lanes exchanges words and has half of the eight bytes.  Tokens side by
// side, as a prompt's are, store v in words of four tokens, others in bytes.
//
// Bound by memory and, as closely, by the issue of 20 vector instructions an element
// (five of them for ties, which a seventh of the rows of bf16 have; with the row
// quantizers' coder, a scale in every lane and loads that waited for one another it was
// 58 us): 30011 tokens of 8 heads of 128 bf16, 156 MB, in 33 to 37 us, 4.2 to 4.7 TB/s;
// float32, 278 MB, in 70.
template <typename T, int LPR, int Q>
__global__ __launch_bounds__(256) void k_kv4_write(KvArgs a)
{
    const int w = threadIdx.x % LPR, words = a.W / 8;
    const uint32_t r = blockIdx.x * (uint32_t)(256 / LPR) + threadIdx.x / LPR;
    if (r >= a.rows) return;
    const bool val = blockIdx.y != 0;
    // four groups after one another have sixteen tokens of a head: a tile's lines are
    // then written by one wave
    const uint32_t u = Q == 4 ? r >> 2 : r, ut = u / (uint32_t)a.H;
    const int h = (int)(u - ut * (uint32_t)a.H);
    const int64_t t0 = Q == 4 ? (int64_t)ut * 16 + (r & 3) * 4 : ut;
    const int nt = (int)(a.T - t0 < Q ? a.T - t0 : Q);
    if (nt <= 0) return;
    const T* x0 = val ? (const T*)a.v + h * a.v_hs : (const T*)a.k + h * a.k_hs;
    const int64_t ld = val ? a.v_ld : a.k_ld;
    Kv8<T> raw[Q];
    const T* from = x0 + t0 * ld + w * 8;
    const int n = a.D - w * 8;
    if (n >= 8) {
#pragma unroll
        for (int q = 0; q < Q; q++, from += q < nt ? ld : 0) raw[q].load(from);
    } else {
#pragma unroll
        for (int q = 0; q < Q; q++, from += q < nt ? ld : 0) raw[q].load(from, n);
    }
    const int m = Q == 4 ? w & 3 : 0;                          // the token that this lane sees to
    int64_t at = m < nt ? kv_slot(a, t0 + m) : -1;
    if (at >= a.n_slots) {
        if (w < Q) set_status(a.status, ISEG_DEV_RANGE);
        at = -1;
    }
    const int32_t slot = at < 0 ? -1 : (int32_t)at;
    const KvPlace p = kv_place(a, slot < 0 ? 0 : slot, h);
    const int nc = a.W / 32;
    const int64_t off = val ? p.tile + (p.t >> 2) * nc * 4 + (p.t & 3) : p.row * (a.W / 2);      // in the codes
    uint32_t big = 0;
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const uint32_t b = kv_max<LPR>(kv_big(raw[q]));
        big = q == 0 || m == q ? b : big;
    }
    const float sm = kv_scale(kv_bits<T>(big), a.mode), im = 1.f / sm;
    if (w < Q && slot >= 0) {
        (val ? a.vs : a.ks)[p.row] = sm;
        if (!(sm == sm)) set_status(a.status, ISEG_DEV_NONFINITE);
    }
    uint32_t x[Q][8];
    int32_t slots[Q];
    int64_t offs[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const float s = __builtin_bit_cast(float, kv_from<Q>(__builtin_bit_cast(uint32_t, sm), q));
        const float inv = __builtin_bit_cast(float, kv_from<Q>(__builtin_bit_cast(uint32_t, im), q));
        slots[q] = (int32_t)kv_from<Q>((uint32_t)slot, q);
        offs[q] = (int64_t)((uint64_t)kv_from<Q>((uint32_t)(off >> 32), q) << 32 | kv_from<Q>((uint32_t)off, q));
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] = raw[q].at(e);
        kv_codes(f, s, inv, x[q]);
        if (!(s == s)) {                                       // zeros
#pragma unroll
            for (int e = 0; e < 8; e++) x[q][e] = 8u << 19;
        }
    }
    if (!val) {
        // even codes in the low half, odd ones in the high half
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const uint32_t word = kv_halves(kv_gather(x[q][0], x[q][4], x[q][1], x[q][5]), kv_gather(x[q][2], x[q][6], x[q][3], x[q][7]));
            if (slots[q] >= 0 && w < words) *(uint32_t*)(a.kc + offs[q] + w * 4) = word;
        }
        return;
    }
    // four tokens' codes of a column; the lane without bit 1 has the low halves'
    // columns, its partner the high ones'
    uint32_t word[4];
    const bool hi = w & 2;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const uint32_t y = Q == 4 ? kv_gather(x[0][e], x[Q / 4][e], x[Q / 2][e], x[Q - 1][e]) : x[0][e] >> 16;
        const uint32_t z = Q == 4 ? kv_gather(x[0][4 + e], x[Q / 4][4 + e], x[Q / 2][4 + e], x[Q - 1][4 + e]) : x[0][4 + e] >> 16;
        const uint32_t give = hi ? y : z, mine = hi ? z : y;
        const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp((int)give, (int)give, 0x4e, 0xf, 0xf, false);
        word[e] = kv_halves(hi ? got : mine, hi ? mine : got);
    }
    if (w >= words) return;
    uint8_t* to = a.vc + ((w & 1) * 8 + ((w & 2) ? 4 : 0)) * 16 * nc + (w >> 2) * 4;
    const int32_t first = slots[0];
    if (Q == 4 && first >= 0 && (first & 3) == 0 && slots[Q / 4] == first + 1 && slots[Q / 2] == first + 2 && slots[Q - 1] == first + 3) {
#pragma unroll
        for (int e = 0; e < 4; e++) *(uint32_t*)(to + offs[0] + 16 * e * nc) = word[e];
        return;
    }
#pragma unroll
    for (int t = 0; t < Q; t++) {
        if (slots[t] < 0) continue;
#pragma unroll
        for (int e = 0; e < 4; e++) to[offs[t] + 16 * e * nc] = (uint8_t)(word[e] >> (8 * t));
    }
}

// whether four tokens lie side by side in one run of four of a tile
__device__ __forceinline__ bool kv_beside(const int64_t* slot, const KvArgs& a)
{
    return slot[0] >= 0 && slot[0] + 3 < a.n_slots && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 &&
           slot[3] == slot[0] + 3;
}

// The same deal the other way: 30011 tokens of 8 heads of 128 to bf16, 156 MB, in 27
// us (5.7 TB/s: the codes come from the last-level cache).
template <typename T, int LPR, int Q>
__global__ __launch_bounds__(256) void k_kv4_read(KvArgs a)
{
    const int w = threadIdx.x % LPR, words = a.W / 8;
    const uint32_t r = blockIdx.x * (uint32_t)(256 / LPR) + threadIdx.x / LPR;
    if (r >= a.rows || w >= words) return;
    const bool val = blockIdx.y != 0;
    // sixteen tokens of a head by four groups after one another, as in the writing
    const uint32_t u = Q == 4 ? r >> 2 : r, ut = u / (uint32_t)a.H;
    const int h = (int)(u - ut * (uint32_t)a.H);
    const int64_t t0 = Q == 4 ? (int64_t)ut * 16 + (r & 3) * 4 : ut;
    const int nt = (int)(a.T - t0 < Q ? a.T - t0 : Q);
    if (nt <= 0) return;
    int64_t slot[Q];
    float s[Q];
    int n[Q][8];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        slot[q] = q < nt ? kv_slot(a, t0 + q) : -1;
        if (slot[q] >= a.n_slots) {
            if (w == 0) set_status(a.status, ISEG_DEV_RANGE);
            slot[q] = -1;
        }
        s[q] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) n[q][e] = 0;
    }
    const int i = w >> 2, c0 = (w & 1) * 8, up = (w & 2) ? 4 : 0, nc = a.W / 32;
    if (!val) {
#pragma unroll
        for (int q = 0; q < Q; q++) {
            if (slot[q] < 0) continue;
            const KvPlace p = kv_place(a, slot[q], h);
            s[q] = a.ks[p.row];
            const uint32_t word = *(const uint32_t*)(a.kc + p.row * (a.W / 2) + w * 4);
#pragma unroll
            for (int e = 0; e < 8; e++) n[q][e] = (int)((word >> ((e & 1) * 16 + (e >> 1) * 4)) & 15u) - 8;
        }
    } else if (Q == 4 && kv_beside(slot, a)) {
        const KvPlace p = kv_place(a, slot[0], h);
        const uint8_t* b = a.vc + p.tile + ((c0 * 4 + (p.t >> 2)) * nc + i) * 4;
        uint32_t word[8];
#pragma unroll
        for (int e = 0; e < 8; e++) word[e] = *(const uint32_t*)(b + 16 * e * nc);
#pragma unroll
        for (int q = 0; q < Q; q++) {
            s[q] = a.vs[p.row + q];
#pragma unroll
            for (int e = 0; e < 8; e++) n[q][e] = (int)((word[e] >> (8 * q + up)) & 15u) - 8;
        }
    } else {
#pragma unroll
        for (int q = 0; q < Q; q++) {
            if (slot[q] < 0) continue;
            const KvPlace p = kv_place(a, slot[q], h);
            s[q] = a.vs[p.row];
            const uint8_t* b = a.vc + p.tile + ((c0 * 4 + (p.t >> 2)) * nc + i) * 4 + (p.t & 3);
#pragma unroll
            for (int e = 0; e < 8; e++) n[q][e] = (int)((b[16 * e * nc] >> up) & 15) - 8;
        }
    }
    T* out = val ? (T*)a.vo + h * a.v_hs : (T*)a.ko + h * a.k_hs;
    const int64_t ld = val ? a.v_ld : a.k_ld;
    const int d = w * 8;
#pragma unroll
    for (int q = 0; q < Q; q++) {
        if (q >= nt) break;
        struct { T v[8]; } o;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            float f = (float)n[q][e] * s[q];
            asm("" : "+v"(f));                                 // float32 first, whatever type follows: not one step to float16
            o.v[e] = (T)f;
        }
        T* to = out + (t0 + q) * ld;
        if (d + 8 <= a.D) {
            __builtin_memcpy(to + d, &o, sizeof(o));
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (d + e < a.D) to[d + e] = o.v[e];
        }
    }
}

int kv_check(const iseg_kv4_geom* g)
{
    if (!g || !is_float_dtype(g->dtype) || (g->slot_dtype != ISEG_I32 && g->slot_dtype != ISEG_I64)) return ISEG_ERR_ARG;
    if (g->T < 0 || g->H < 0 || g->D < 1 || g->T >= (int64_t)1 << 31 || g->page < 16 || g->page % 16 || g->n_pages < 0)
        return ISEG_ERR_SHAPE;
    if (g->D > 256 || g->page > 8192 || g->H > 65536 || !kv4_pages_ok(g->n_pages, g->page)) return ISEG_ERR_UNSUPPORTED;
    return ISEG_OK;
}

KvArgs kv_args(const iseg_kv4_geom* g, const void* slots, int32_t* status)
{
    KvArgs a = {};
    a.slots = slots; a.T = g->T;
    // one token a group of lanes until there are groups of four for the whole card (8
    // heads of 128 bf16, writing and reading: 64 tokens 3.9 + 3.2 us against 5.1 + 4.2, 512
    // 4.8 + 3.6 against 5.2 + 4.6, 2048 8.4 + 6.3 against 5.9 + 5.4, 30011 69 + 45 against
    // 33 + 27)
    a.four = g->T * g->H >= 8192;
    a.rows = a.four ? ceil_div64(g->T, 16) * 4 * g->H : g->T * g->H;
    a.k_ld = g->k_ld; a.k_hs = g->k_hs; a.v_ld = g->v_ld; a.v_hs = g->v_hs;
    a.n_slots = g->n_pages * g->page; a.H = (int32_t)g->H; a.D = (int32_t)g->D; a.W = kv4_width(g->D); a.page = g->page;
    a.slot64 = g->slot_dtype == ISEG_I64; a.mode = g->scale_mode; a.status = status;
    return a;
}

#define KV_LAUNCH(kernel, LPR)                                                                                   \
    do {                                                                                                         \
        const dim3 grid((unsigned)ceil_div64(a.rows, 256 / LPR), 2);                                             \
        if (a.four) hipLaunchKernelGGL((kernel<T, LPR, 4>), grid, dim3(256), 0, s, a);                           \
        else hipLaunchKernelGGL((kernel<T, LPR, 1>), grid, dim3(256), 0, s, a);                                  \
    } while (0)

template <typename T>
int kv_write(const KvArgs& a, hipStream_t s)
{
    if (a.W <= 32) KV_LAUNCH(k_kv4_write, 4);
    else if (a.W <= 64) KV_LAUNCH(k_kv4_write, 8);
    else if (a.W <= 128) KV_LAUNCH(k_kv4_write, 16);
    else KV_LAUNCH(k_kv4_write, 32);
    return launch_ok();
}

template <typename T>
int kv_read(const KvArgs& a, hipStream_t s)
{
    if (a.W <= 32) KV_LAUNCH(k_kv4_read, 4);
    else if (a.W <= 64) KV_LAUNCH(k_kv4_read, 8);
    else if (a.W <= 128) KV_LAUNCH(k_kv4_read, 16);
    else KV_LAUNCH(k_kv4_read, 32);
    return launch_ok();
}

// ---------------------------------------------------------------------------
// pages, slots and positions of a step
// ---------------------------------------------------------------------------
struct PmArgs {
    const int32_t *ctx, *count, *free_pages;
    const int32_t *held, *n_free;
    int32_t *table, *q_start, *kv_len, *pos, *slots, *held_out, *n_free_out;
    int32_t *w_held, *w_first, *w_free;       // workspace: pages held before, first page taken, free pages before
    int64_t T, max_pages, table_ld, F, n_pages;
    int32_t B, page;
    int32_t lanes;                   // 2^lanes threads write a request's new pages
    int32_t* status;
};

// inclusive sums of two values over the block's 1024 threads
__device__ __forceinline__ void scan2_1024(int64_t& x, int64_t& y, int64_t (*red)[16])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(x, o, 64), v = __shfl_up(y, o, 64);
        if (lane >= o) { x += u; y += v; }
    }
    __syncthreads();
    if (lane == 63) { red[0][w] = x; red[1][w] = y; }
    __syncthreads();
    for (int i = 0; i < w; i++) { x += red[0][i]; y += red[1][i]; }
}

__device__ __forceinline__ int32_t sat31(int64_t v) { return (int32_t)(v < 0x7fffffff ? v : 0x7fffffff); }

// Pages of a step.  There is next to nothing to move (256 requests: 6 KB); what counts
// is the chain lengths -> sums -> page taken -> slot, each link a trip to memory.
//
// by one block: lengths, pages wanted, their sums; `near` (LDS, or NULL) gets q_start
// as well
__device__ __forceinline__ void page_scan(const PmArgs& a, int32_t* near)
{
    __shared__ int64_t red[2][16];
    __shared__ int64_t base[2];
    int bad = 0;
    int64_t nf = *a.n_free;
    if (nf < 0 || nf > a.F) { bad = 1; nf = nf < 0 ? 0 : a.F; }
    if (threadIdx.x == 0) { base[0] = base[1] = 0; }
    __syncthreads();
    for (int32_t b0 = 0; b0 < a.B; b0 += 1024) {
        const int32_t b = b0 + (int32_t)threadIdx.x;
        int64_t n = 0, need = 0, first_t, first_p;
        int32_t held = 0;
        if (b < a.B) {
            int64_t c = a.ctx[b];
            n = a.count[b];
            held = a.held[b];
            if (c < 0 || n < 0 || held < 0 || held > a.max_pages) bad = 1;
            c = c < 0 ? 0 : c;
            n = n < 0 ? 0 : n;
            held = held < 0 ? 0 : (held > a.max_pages ? (int32_t)a.max_pages : held);
            const int64_t kv = c + n;
            int64_t want = (kv + a.page - 1) / a.page;
            if (want > a.max_pages) { bad = 1; want = a.max_pages; }
            need = want > held ? want - held : 0;
            if (kv > 0x7fffffff) bad = 1;
            a.kv_len[b] = sat31(kv);
        }
        int64_t sn = n, sp = need;
        scan2_1024(sn, sp, red);
        first_t = base[0] + sn - n;
        first_p = base[1] + sp - need;
        if (b < a.B) {
            a.q_start[b] = sat31(first_t);
            if (near) near[b] = sat31(first_t);
            a.w_held[b] = held;
            a.w_first[b] = sat31(first_p);
            const int64_t got = nf - first_p < 0 ? 0 : (nf - first_p < need ? nf - first_p : need);
            if (got < need) bad = 1;
            a.held_out[b] = held + (int32_t)got;
        }
        __syncthreads();
        if (threadIdx.x == 1023) { base[0] += sn; base[1] += sp; }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        if (base[0] > a.T) bad = 1;
        a.q_start[a.B] = sat31(base[0]);
        if (near) near[a.B] = sat31(base[0]);
        *a.w_free = (int32_t)nf;
        *a.n_free_out = (int32_t)(nf > base[1] ? nf - base[1] : 0);
    }
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
}

// entry k of the free list as a page; -1: none
__device__ __forceinline__ int32_t page_taken(const PmArgs& a, int64_t k, int& bad)
{
    const int32_t pg = k >= 0 ? a.free_pages[k] : -1;
    if (pg >= 0 && pg < a.n_pages) return pg;
    bad = 1;
    return -1;
}

// page of column `col` of request b: taken now, or in the table already; -1: none
__device__ __forceinline__ int32_t page_of(const PmArgs& a, int32_t b, int64_t col, int& bad)
{
    if (col >= a.max_pages) { bad = 1; return -1; }
    const int32_t held = a.w_held[b];
    int32_t pg = -1;
    if (col < held) {
        pg = a.table[(int64_t)b * a.table_ld + col];
    } else {
        return page_taken(a, (int64_t)*a.w_free - 1 - a.w_first[b] - (col - held), bad);
    }
    if (pg < 0 || pg >= a.n_pages) { bad = 1; pg = -1; }
    return pg;
}

// request of a row of the step: the last b with q_start[b] <= row
__device__ __forceinline__ int32_t request_of(const int32_t* start, int32_t B, int64_t row)
{
    int32_t lo = 0, hi = B;                       // start[lo] <= row < start[hi]
    while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (start[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// tokens and then requests, dealt to `blocks` blocks of NT threads: a thread per
// token, a few threads per request for the pages that it takes.  start: q_start, in LDS
// where it fits, since the search for a token's request is a chain of reads
template <int NT>
__device__ __forceinline__ void page_fill(const PmArgs& a, const int32_t* start, int64_t block, int64_t blocks)
{
    const int64_t total = start[a.B];
    int bad = 0;
    for (int64_t r = block * NT + threadIdx.x; r < a.T; r += blocks * NT) {
        if (r >= total) {
            a.pos[r] = 0;
            a.slots[r] = -1;
            continue;
        }
        const int32_t b = request_of(start, a.B, r);
        const int64_t c = a.ctx[b] < 0 ? 0 : a.ctx[b], p = c + (r - start[b]);
        const int64_t col = p / a.page;
        const int32_t pg = page_of(a, b, col, bad), in = (int32_t)(p - col * a.page);
        a.pos[r] = sat31(p);
        a.slots[r] = pg < 0 ? -1 : pg * a.page + in;
    }
    const int64_t free = *a.w_free;
    for (int64_t r = block * NT + threadIdx.x; r < (int64_t)a.B << a.lanes; r += blocks * NT) {
        const int64_t b = r >> a.lanes;
        const int64_t c = a.ctx[b] < 0 ? 0 : a.ctx[b], n = a.count[b] < 0 ? 0 : a.count[b], held = a.w_held[b], first = a.w_first[b];
        int64_t want = (c + n + a.page - 1) / a.page;
        if (want > a.max_pages) want = a.max_pages;
        for (int64_t col = held + (r & ((1 << a.lanes) - 1)); col < want; col += (int64_t)1 << a.lanes)
            a.table[b * a.table_ld + col] = page_taken(a, free - 1 - first - (col - held), bad);
    }
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
}

constexpr int kStarts = 4096;              // requests whose first rows LDS holds

__global__ __launch_bounds__(1024) void k_page_scan(PmArgs a) { page_scan(a, nullptr); }

__global__ __launch_bounds__(256) void k_page_fill(PmArgs a)
{
    __shared__ int32_t near[kStarts + 1];
    if (a.B <= kStarts) {
        for (int32_t b = threadIdx.x; b <= a.B; b += 256) near[b] = a.q_start[b];
        __syncthreads();
    }
    page_fill<256>(a, a.B <= kStarts ? near : a.q_start, blockIdx.x, gridDim.x);
}

// a decoding step: both in one block, whose own writes to the workspace the barrier
// makes visible to it
__global__ __launch_bounds__(1024) void k_page_map(PmArgs a)
{
    __shared__ int32_t near[1025];
    page_scan(a, near);
    __syncthreads();
    page_fill<1024>(a, near, 0, 1);
}

int pm_check(const iseg_page_map_geom* g)
{
    if (!g || g->reserved) return ISEG_ERR_ARG;
    if (g->B < 0 || g->T < 0 || g->B >= ((int64_t)1 << 31) - 1 || g->T >= (int64_t)1 << 31 || g->max_pages < 0 ||
        g->table_ld < g->max_pages || g->F < 0 || g->n_pages < 0 || g->page < 1)
        return ISEG_ERR_SHAPE;
    if (!kv4_pages_ok(g->n_pages, g->page) || g->max_pages >= (int64_t)1 << 31 || g->F >= (int64_t)1 << 31)
        return ISEG_ERR_UNSUPPORTED;
    return ISEG_OK;
}

}  // namespace

extern "C" int iseg_kv4_write(const void* k, const void* v, const void* slots, const iseg_kv4_geom* g,
                              uint8_t* k_codes, float* k_scale, uint8_t* v_codes, float* v_scale,
                              int32_t* dev_status, hipStream_t stream)
{
    const int rc = kv_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->scale_mode != ISEG_SCALE_MAX && g->scale_mode != ISEG_SCALE_POW2) return ISEG_ERR_ARG;
    if (g->k_ld < 0 || g->k_hs < 0 || g->v_ld < 0 || g->v_hs < 0) return ISEG_ERR_SHAPE;
    if (g->T == 0 || g->H == 0) return ISEG_OK;
    if (!k || !v || !slots || (g->n_pages > 0 && (!k_codes || !k_scale || !v_codes || !v_scale))) return ISEG_ERR_ARG;
    if (((uintptr_t)k_codes | (uintptr_t)v_codes) & 15) return ISEG_ERR_ARG;
    KvArgs a = kv_args(g, slots, dev_status);
    if (ceil_div64(a.rows, 8) >= (int64_t)1 << 24) return ISEG_ERR_UNSUPPORTED;
    a.k = k; a.v = v; a.kc = k_codes; a.ks = k_scale; a.vc = v_codes; a.vs = v_scale;
    return g->dtype == ISEG_F32 ? kv_write<float>(a, stream)
                                : g->dtype == ISEG_F16 ? kv_write<f16_t>(a, stream) : kv_write<bf16_t>(a, stream);
}

extern "C" int iseg_kv4_read(const uint8_t* k_codes, const float* k_scale, const uint8_t* v_codes,
                             const float* v_scale, const void* slots, const iseg_kv4_geom* g, void* k, void* v,
                             int32_t* dev_status, hipStream_t stream)
{
    const int rc = kv_check(g);
    if (rc != ISEG_OK) return rc;
    if (!rows_apart(g->T, g->H, g->D, g->k_ld, g->k_hs) || !rows_apart(g->T, g->H, g->D, g->v_ld, g->v_hs))
        return ISEG_ERR_SHAPE;
    if (g->T == 0 || g->H == 0) return ISEG_OK;
    if (!k || !v || !slots || (g->n_pages > 0 && (!k_codes || !k_scale || !v_codes || !v_scale))) return ISEG_ERR_ARG;
    if (((uintptr_t)k_codes | (uintptr_t)v_codes) & 15) return ISEG_ERR_ARG;
    KvArgs a = kv_args(g, slots, dev_status);
    if (ceil_div64(a.rows, 8) >= (int64_t)1 << 24) return ISEG_ERR_UNSUPPORTED;
    a.ko = k; a.vo = v; a.kc = (uint8_t*)k_codes; a.ks = (float*)k_scale; a.vc = (uint8_t*)v_codes;
    a.vs = (float*)v_scale;
    return g->dtype == ISEG_F32 ? kv_read<float>(a, stream)
                                : g->dtype == ISEG_F16 ? kv_read<f16_t>(a, stream) : kv_read<bf16_t>(a, stream);
}

extern "C" size_t iseg_page_map_ws(const iseg_page_map_geom* g)
{
    if (pm_check(g) != ISEG_OK) return 0;
    return ws_used(align256((size_t)g->B * 4) * 2 + 256);
}

extern "C" int iseg_page_map(const int32_t* ctx, const int32_t* count, const int32_t* held, const int32_t* free_pages,
                             const int32_t* n_free, const iseg_page_map_geom* g, int32_t* table, int32_t* q_start,
                             int32_t* kv_len, int32_t* positions, int32_t* slots, int32_t* held_out,
                             int32_t* n_free_out, void* ws, size_t ws_bytes, int32_t* dev_status, hipStream_t stream)
{
    const int rc = pm_check(g);
    if (rc != ISEG_OK) return rc;
    if (!n_free || !n_free_out || !q_start || (g->F > 0 && !free_pages) || (g->T > 0 && (!positions || !slots)))
        return ISEG_ERR_ARG;
    if (g->B > 0 && (!ctx || !count || !held || !kv_len || !held_out || (g->max_pages > 0 && !table))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_page_map_ws(g)) return ISEG_ERR_WORKSPACE;
    PmArgs a = {};
    a.ctx = ctx; a.count = count; a.held = held; a.free_pages = free_pages; a.n_free = n_free;
    a.table = table; a.q_start = q_start; a.kv_len = kv_len; a.pos = positions; a.slots = slots;
    a.held_out = held_out; a.n_free_out = n_free_out;
    a.w_held = (int32_t*)ws;
    a.w_first = (int32_t*)((char*)ws + align256((size_t)g->B * 4));
    a.w_free = (int32_t*)((char*)ws + 2 * align256((size_t)g->B * 4));
    a.T = g->T; a.max_pages = g->max_pages; a.table_ld = g->table_ld; a.F = g->F; a.n_pages = g->n_pages;
    a.B = (int32_t)g->B; a.page = g->page; a.status = dev_status;
    // threads for about as many pages as a request takes on average, and the first few
    const int64_t pages = g->B > 0 ? g->T / g->B / g->page : 0;
    a.lanes = 2;
    while (a.lanes < 6 && (1 << a.lanes) < pages) a.lanes++;
    // up to 4096 tokens of 1024 requests by one block: a launch less for the host (about
    // 4 us), and captured 256 requests of one token 5.7 us against 7.2, 1000 8.4 against
    // 9.3, 900 of four 11.7 against 9.6
    if (g->T <= 4096 && g->B <= 1024) {
        hipLaunchKernelGGL(k_page_map, dim3(1), dim3(1024), 0, stream, a);
    } else {
        hipLaunchKernelGGL(k_page_scan, dim3(1), dim3(1024), 0, stream, a);
        const int64_t fill = g->B << a.lanes, items = ceil_div64(g->T > fill ? g->T : fill, 256);
        hipLaunchKernelGGL(k_page_fill, dim3((unsigned)(items < 2048 ? items : 2048)), dim3(256), 0, stream, a);
    }
    return launch_ok();
}
