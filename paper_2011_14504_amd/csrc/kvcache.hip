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

// eight elements of a row from d on, zeros beyond D
template <typename T>
__device__ __forceinline__ void kv_get8(const T* p, int d, int D, float* f)
{
    if (d + 8 <= D) {
        struct { T v[8]; } r;
        __builtin_memcpy(&r, p + d, sizeof(r));
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = (float)r.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = d + i < D ? (float)p[d + i] : 0.f;
    }
}

// Scale of a largest magnitude given as float32 bits: scale_of (coder.h) with 4
// bits, in float32.  A float32 quotient rounded once is the float64 one rounded to
// float32 (24 bits twice and two more fit in 53).  In float64 the write of 30011
// tokens takes 2 us more.
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

// whether four tokens lie side by side in one run of four of a tile
__device__ __forceinline__ bool kv_beside(const int64_t* slot, const KvArgs& a)
{
    return slot[0] >= 0 && slot[0] + 3 < a.n_slots && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 &&
           slot[3] == slot[0] + 3;
}

// LPR lanes a row, eight columns (a word of codes) a lane, four tokens of a head
// at a time; blockIdx.y: keys or values.  The largest magnitude over the row's
// lanes, the scale, the codes.  A byte of v holds columns 16 apart, which lie two
// lanes apart: each pair of lanes exchanges words and has half of the eight
// bytes.  Tokens side by side, as a prompt's are, store v in words of four
// tokens, others in bytes.
template <typename T, int LPR, int Q>
__global__ __launch_bounds__(256) void k_kv4_write(KvArgs a)
{
    const int w = threadIdx.x % LPR, words = a.W / 8;
    const int64_t r = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    if (r >= a.rows) return;
    const bool val = blockIdx.y != 0;
    // four groups after one another have sixteen tokens of a head: a tile's lines are
    // then written by one wave
    const int64_t u = Q == 4 ? r >> 2 : r, ut = u / a.H;
    const int h = (int)(u - ut * a.H);
    const int64_t t0 = Q == 4 ? ut * 16 + (r & 3) * 4 : ut;
    const int nt = (int)(a.T - t0 < Q ? a.T - t0 : Q);
    if (nt <= 0) return;
    const T* x0 = val ? (const T*)a.v + h * a.v_hs : (const T*)a.k + h * a.k_hs;
    const int64_t ld = val ? a.v_ld : a.k_ld;
    int64_t slot[Q];
    float f[Q][8];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        slot[q] = q < nt ? kv_slot(a, t0 + q) : -1;
        if (slot[q] >= a.n_slots) {
            if (w == 0) set_status(a.status, ISEG_DEV_RANGE);
            slot[q] = -1;
        }
    }
#pragma unroll
    for (int q = 0; q < Q; q++) kv_get8(x0 + (t0 + (q < nt ? q : 0)) * ld, w * 8, a.D, f[q]);
    uint32_t bytes[Q];                                         // v: of each token
#pragma unroll
    for (int q = 0; q < Q; q++) {
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t b = bits_of(f[q][i]);
            big = b > big ? b : big;
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) {
            const uint32_t b = (uint32_t)__shfl_xor((int)big, o, 64);
            big = b > big ? b : big;
        }
        const Coder cd(kv_scale(big, a.mode));
        const float s = cd.s;
        uint32_t n[2];
        codes_of<8, false>(f[q], nullptr, [&](int) -> const Coder& { return cd; }, 7, n);
        if (!cd.ok) {
            n[0] = n[1] = 0;
            if (w == 0 && slot[q] >= 0) set_status(a.status, ISEG_DEV_NONFINITE);
        }
        // bytes n in [-7, 7] to n + 8
        n[0] = (n[0] & 0x0f0f0f0fu) ^ 0x08080808u;
        n[1] = (n[1] & 0x0f0f0f0fu) ^ 0x08080808u;
        if (!val) {
            if (slot[q] < 0) continue;
            const KvPlace p = kv_place(a, slot[q], h);
            // even codes in the low half, odd ones in the high half
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) word |= ((n[e >> 2] >> (8 * (e & 3))) & 15u) << ((e & 1) * 16 + (e >> 1) * 4);
            if (w < words) *(uint32_t*)(a.kc + p.row * (a.W / 2) + w * 4) = word;
            if (w == 0) a.ks[p.row] = s;
        } else {
            // the lane without bit 1 has the low halves' columns, its partner the high ones'
            const bool hi = w & 2;
            const uint32_t give = hi ? n[0] : n[1], mine = hi ? n[1] : n[0];
            const uint32_t got = (uint32_t)__shfl_xor((int)give, 2, 64);
            bytes[q] = hi ? got | mine << 4 : mine | got << 4;
            if (w == 0 && slot[q] >= 0) a.vs[kv_place(a, slot[q], h).row] = s;
        }
    }
    if (!val || w >= words) return;
    const int i = w >> 2, c0 = (w & 1) * 8 + ((w & 2) ? 4 : 0), nc = a.W / 32;
    if constexpr (Q == 4) if (kv_beside(slot, a)) {
        const KvPlace p = kv_place(a, slot[0], h);
        uint8_t* q = a.vc + p.tile + ((c0 * 4 + (p.t >> 2)) * nc + i) * 4;
        // four tokens' bytes of four columns to four columns' bytes of four tokens
        const uint32_t lo01 = __builtin_amdgcn_perm(bytes[1], bytes[0], 0x05010400), lo23 = __builtin_amdgcn_perm(bytes[3], bytes[2], 0x05010400);
        const uint32_t hi01 = __builtin_amdgcn_perm(bytes[1], bytes[0], 0x07030602), hi23 = __builtin_amdgcn_perm(bytes[3], bytes[2], 0x07030602);
        *(uint32_t*)(q) = __builtin_amdgcn_perm(lo23, lo01, 0x05040100);
        *(uint32_t*)(q + 16 * nc) = __builtin_amdgcn_perm(lo23, lo01, 0x07060302);
        *(uint32_t*)(q + 32 * nc) = __builtin_amdgcn_perm(hi23, hi01, 0x05040100);
        *(uint32_t*)(q + 48 * nc) = __builtin_amdgcn_perm(hi23, hi01, 0x07060302);
        return;
    }
#pragma unroll
    for (int t = 0; t < Q; t++) {
        if (slot[t] < 0) continue;
        const KvPlace p = kv_place(a, slot[t], h);
        uint8_t* q = a.vc + p.tile + ((c0 * 4 + (p.t >> 2)) * nc + i) * 4 + (p.t & 3);
#pragma unroll
        for (int e = 0; e < 4; e++) q[16 * e * nc] = (uint8_t)(bytes[t] >> (8 * e));
    }
}

template <typename T, int LPR, int Q>
__global__ __launch_bounds__(256) void k_kv4_read(KvArgs a)
{
    const int w = threadIdx.x % LPR, words = a.W / 8;
    const int64_t r = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    if (r >= a.rows || w >= words) return;
    const bool val = blockIdx.y != 0;
    // four groups after one another have sixteen tokens of a head: a tile's lines are
    // then written by one wave
    const int64_t u = Q == 4 ? r >> 2 : r, ut = u / a.H;
    const int h = (int)(u - ut * a.H);
    const int64_t t0 = Q == 4 ? ut * 16 + (r & 3) * 4 : ut;
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
        for (int e = 0; e < 8; e++) o.v[e] = (T)((float)n[q][e] * s[q]);
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
    // one token a group of lanes until there are groups of four for the whole card:
    // 64 tokens of 8 heads 4.0 us against 8.5, 30011 tokens 64 against 78
    a.four = g->T * g->H >= 4096;
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

// by one block: lengths, pages wanted, their sums
__device__ __forceinline__ void page_scan(const PmArgs& a)
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
        *a.w_free = (int32_t)nf;
        *a.n_free_out = (int32_t)(nf > base[1] ? nf - base[1] : 0);
    }
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
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
        const int64_t k = (int64_t)*a.w_free - 1 - a.w_first[b] - (col - held);
        if (k >= 0) pg = a.free_pages[k];
        else bad = 1;
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
// token; a wave per request for the pages that it takes
template <int NT>
__device__ __forceinline__ void page_fill(const PmArgs& a, int64_t block, int64_t blocks)
{
    const int64_t total = a.q_start[a.B];
    int bad = 0;
    for (int64_t r = block * NT + threadIdx.x; r < a.T; r += blocks * NT) {
        if (r >= total) {
            a.pos[r] = 0;
            a.slots[r] = -1;
            continue;
        }
        const int32_t b = request_of(a.q_start, a.B, r);
        const int64_t c = a.ctx[b] < 0 ? 0 : a.ctx[b], p = c + (r - a.q_start[b]);
        const int64_t col = p / a.page;
        const int32_t pg = page_of(a, b, col, bad), in = (int32_t)(p - col * a.page);
        a.pos[r] = sat31(p);
        a.slots[r] = pg < 0 ? -1 : pg * a.page + in;
    }
    for (int64_t b = block * (NT / 64) + (threadIdx.x >> 6); b < a.B; b += blocks * (NT / 64)) {
        const int64_t c = a.ctx[b] < 0 ? 0 : a.ctx[b], n = a.count[b] < 0 ? 0 : a.count[b];
        int64_t want = (c + n + a.page - 1) / a.page;
        if (want > a.max_pages) want = a.max_pages;
        for (int64_t col = a.w_held[b] + (int64_t)(threadIdx.x & 63); col < want; col += 64)
            a.table[b * a.table_ld + col] = page_of(a, (int32_t)b, col, bad);
    }
    if (bad) set_status(a.status, ISEG_DEV_RANGE);
}

__global__ __launch_bounds__(1024) void k_page_scan(PmArgs a) { page_scan(a); }

__global__ __launch_bounds__(256) void k_page_fill(PmArgs a) { page_fill<256>(a, blockIdx.x, gridDim.x); }

// a decoding step: both in one block, whose own writes to q_start and the
// workspace the barrier makes visible to it
__global__ __launch_bounds__(1024) void k_page_map(PmArgs a)
{
    page_scan(a);
    __syncthreads();
    page_fill<1024>(a, 0, 1);
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
    // up to 4096 tokens of 1024 requests the one block takes no longer than a second
    // launch (256 requests of one token: 6 us, and 5 + 3 in two)
    if (g->T <= 4096 && g->B <= 1024) {
        hipLaunchKernelGGL(k_page_map, dim3(1), dim3(1024), 0, stream, a);
    } else {
        hipLaunchKernelGGL(k_page_scan, dim3(1), dim3(1024), 0, stream, a);
        const int64_t items = ceil_div64(g->T, 256) > ceil_div64(g->B, 4) ? ceil_div64(g->T, 256) : ceil_div64(g->B, 4);
        hipLaunchKernelGGL(k_page_fill, dim3((unsigned)(items < 2048 ? items : 2048)), dim3(256), 0, stream, a);
    }
    return launch_ok();
}
