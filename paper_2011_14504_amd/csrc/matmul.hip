// matmul.hip -- int8 x int8 matrix products on MFMA with a scale for each row
// of either operand (iseg_matmul_i8).
//
// Both operands have the reduction along the row, so a 16-byte piece of a row
// is one lane's operand of v_mfma_i32_16x16x64_i8.  The int32 sums are exact,
// so any split of the reduction gives the same bits.
#include "coder.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

struct MmArgs {
    const int8_t *a, *b;
    const float *sa, *sb, *bias;
    void* out;
    int64_t M, N, K, lda, ldb, ldc;
    uint32_t tm, tn;             // tiles
    int64_t ksplit;              // reduction of one split (a multiple of 128)
    int64_t ldc_part;            // rows of the splits' sums (N rounded up to 4)
};

template <typename TO>
struct alignas(4 * sizeof(TO)) OutVec {
    TO v[4];
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

// 16 bytes from p + k of a row that starts off a multiple of four: five whole
// words, shifted (11 x 4160 x 14279: 62 us with loads at odd bytes, 36 so).
// Touches up to three bytes before p + k and after its 16.
__device__ __forceinline__ v4i load16_odd(const int8_t* p, int64_t k)
{
    const uint32_t sh = (uint32_t)((uintptr_t)p & 3);
    const uint32_t* q = (const uint32_t*)(p - sh + k);
    uint32_t d[5];
    __builtin_memcpy(d, __builtin_assume_aligned(q, 4), 16);
    d[4] = q[4];
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = (int)__builtin_amdgcn_alignbyte(d[i + 1], d[i], sh);
    return r;
}

// An output from its sum: two roundings after the sum's own, the same in every
// kernel, so a row has the same bits alone and in a batch.
__device__ __forceinline__ float mm_out(int sum, float sa, float sb, float bias)
{
    return fmaf((float)sum * sa, sb, bias);
}

// the fragment of the last K % 16 columns: zero but for the first 16 bytes of
// the reduction step (lp = 0)
__device__ __forceinline__ v4i mm_tail(const int8_t* x, int64_t ld, int64_t row, int64_t rows, int64_t K, int lp)
{
    const v4i z = {0, 0, 0, 0};
    return lp == 0 && row < rows ? load16(x + row * ld, K & ~(int64_t)15, K) : z;
}

// byte of a 16-byte piece in an LDS tile of 128-byte rows: the pieces of a row
// are turned by half the row's number, which spreads the 16 rows of a fragment
// read over the banks
__device__ __forceinline__ int mm_swz(int row, int part) { return row * 128 + ((part ^ ((row >> 1) & 7)) << 4); }

// ---------------------------------------------------------------------------
// tiles with direct-to-LDS loads
// ---------------------------------------------------------------------------
typedef __attribute__((address_space(3))) void lds_ptr_t;
__device__ __attribute__((aligned(64))) int8_t g_mm_zero[64];

__device__ __forceinline__ void mm_dma16(const void* g, int8_t* lds_wave_base)
{
    __builtin_amdgcn_global_load_lds(g, (lds_ptr_t*)lds_wave_base, 16, 0, 0);
}

// wait until at most VM loads of this wave are outstanding and its LDS reads are done
template <int VM>
__device__ __forceinline__ void mm_wait()
{
    static_assert(VM >= 0 && VM < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | (7 << 4));
}

// the tile (row, column) of a block: the blocks of one XCD (dealt round-robin
// over 8) take a contiguous run of tiles, walked in bands of 8 rows, so the
// tiles that run at one time on an XCD share rows of a and b in its L2
__device__ __forceinline__ void mm_tile(uint32_t bid, uint32_t tm, uint32_t tn, uint32_t& im, uint32_t& in)
{
    const uint32_t T = tm * tn, q = T >> 3, r = T & 7, x = bid & 7, i = bid >> 3;
    const uint32_t t = x * q + (x < r ? x : r) + i;
    const uint32_t band = 8 * tn, b = t / band, first = b * 8, h = tm - first < 8 ? tm - first : 8;
    const uint32_t u = t - b * band;
    im = first + u % h;
    in = u / h;
}

// BM x BN outputs per block of WM x WN waves, 128 of the reduction per stage
// (whole cache lines of every row), ST stages of LDS.  Large products are bound
// by the matrix cores at the clock that their power leaves: 8192 x 8192 x 8192
// bf16 out 405 to 445 us back to back, by box (2.5 to 2.7 POP/s; 488 to 517 under
// the profiler, where the matrix cores are busy for 64 % of the cycles; zeros as
// operands 349), 4096 x 4096 x 4096 61 (2.25),
// 2048 x 8192 x 2048 36.8 (1.9, one round of 256 tiles, whose epilogues write
// 33 MB at once); small ones by the latency of a stage: 1024 x 2048 x 2048 9.9.
// Eight waves of 128 x 64 outputs, not four of 128 x 128, whose accumulators
// moved between register files (763 us at 8192 against 541 at the time).
template <typename TO, int BM, int BN, int WM, int WN, int ST>
__global__ __launch_bounds__(WM * WN * 64) void k_mm_tile(MmArgs p)
{
    constexpr int NW = WM * WN;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int NA = BM / 8 / NW, NB = BN / 8 / NW, LPW = NA + NB;
    constexpr int SA = BM * 128, SB = BN * 128;
    constexpr bool kSplit = sizeof(TO) == 4 && (TO)0.5f == (TO)0;      // int32 sums of a part of the reduction
    static_assert(NW % 2 == 0, "a lane's piece is the same in all its loads");
    extern __shared__ __attribute__((aligned(16))) int8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t im, in;
    mm_tile(blockIdx.x, p.tm, p.tn, im, in);
    const int64_t m0 = (int64_t)im * BM, n0 = (int64_t)in * BN;
    if constexpr (kSplit) {                   // this split's part of the reduction
        const int64_t k0 = (int64_t)blockIdx.y * p.ksplit;
        p.a += k0;
        p.b += k0;
        p.K = p.K - k0 < p.ksplit ? p.K - k0 : p.ksplit;
        p.out = (int32_t*)p.out + (int64_t)blockIdx.y * p.M * p.ldc;
    }
    const int K16 = (int)p.K & ~15;
    const int kfull = K16 / 128, nk = (K16 + 127) / 128;

    // this lane's pieces: row 8 * instruction + lane / 8 of the tile in slot
    // lane % 8; rows past the end repeat the last one (their outputs are dropped)
    const int rin = lane >> 3, part = (lane & 7) ^ (4 * (wave & 1) + (rin >> 1));
    const int8_t *ap[NA], *bp[NB];
#pragma unroll
    for (int j = 0; j < NA; j++) {
        const int64_t r = m0 + 8 * (wave + NW * j) + rin;
        ap[j] = p.a + (r < p.M ? r : p.M - 1) * p.lda + part * 16;
    }
#pragma unroll
    for (int j = 0; j < NB; j++) {
        const int64_t r = n0 + 8 * (wave + NW * j) + rin;
        bp[j] = p.b + (r < p.N ? r : p.N - 1) * p.ldb + part * 16;
    }
    auto issue = [&](int kb) {
        int8_t* st = smem + (kb % ST) * (SA + SB);
#pragma unroll
        for (int j = 0; j < NA; j++) mm_dma16(ap[j] + kb * 128, st + (wave + NW * j) * 1024);
#pragma unroll
        for (int j = 0; j < NB; j++) mm_dma16(bp[j] + kb * 128, st + SA + (wave + NW * j) * 1024);
    };
    auto issue_end = [&](int kb) {            // zeros past the last whole 16-byte piece
        int8_t* st = smem + (kb % ST) * (SA + SB);
        const bool live = kb * 128 + part * 16 < K16;
#pragma unroll
        for (int j = 0; j < NA; j++)
            mm_dma16(live ? (const void*)(ap[j] + kb * 128) : (const void*)g_mm_zero, st + (wave + NW * j) * 1024);
#pragma unroll
        for (int j = 0; j < NB; j++)
            mm_dma16(live ? (const void*)(bp[j] + kb * 128) : (const void*)g_mm_zero,
                     st + SA + (wave + NW * j) * 1024);
    };

    const int wm = wave / WN, wn = wave % WN;
    const int lr = lane & 15, lp = lane >> 4;
    v4i acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = (v4i){0, 0, 0, 0};
    // fragments of half h (64 of the reduction) of a stage
    auto frags = [&](int kb, int h, v4i* fa, v4i* fb) {
        const int8_t* A = smem + (kb % ST) * (SA + SB);
        const int8_t* B = A + SA;
#pragma unroll
        for (int j = 0; j < TN; j++) fb[j] = *(const v4i*)&B[mm_swz(wn * (TN * 16) + j * 16 + lr, h * 4 + lp)];
#pragma unroll
        for (int i = 0; i < TM; i++) fa[i] = *(const v4i*)&A[mm_swz(wm * (TM * 16) + i * 16 + lr, h * 4 + lp)];
    };
    // b's fragment first: a lane then holds four neighbouring columns of one row
    auto mma = [&](const v4i* fa, const v4i* fb) {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    };
    v4i fa[2][TM], fb[2][TN];
    // one stage: while its first half is multiplied its second half is read;
    // then stage kb + 1 becomes visible and stage kb's buffer free (its reads
    // are done in every wave), and under the second half's products the next
    // loads go out and the next fragments are read
    auto stage = [&](int kb, auto&& issue_next) {
        frags(kb, 1, fa[1], fb[1]);
        mma(fa[0], fb[0]);
        __builtin_amdgcn_sched_barrier(0);
        mm_wait<(ST - 2) * LPW>();
        __builtin_amdgcn_s_barrier();
        issue_next(kb + ST);
        frags(kb + 1, 0, fa[0], fb[0]);
        mma(fa[1], fb[1]);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (nk > 0) {
#pragma unroll
        for (int i = 0; i < ST; i++) issue_end(i);
        mm_wait<(ST - 1) * LPW>();
        __builtin_amdgcn_s_barrier();
        frags(0, 0, fa[0], fb[0]);
        int kb = 0;
        for (; kb + ST < kfull; kb++) stage(kb, issue);
        for (; kb < nk; kb++) stage(kb, issue_end);
        mm_wait<0>();                         // the zeros still on their way to LDS
    }
    if (p.K & 15) {
        // the last 1 to 15 of the reduction straight into the fragments
        const int64_t ra = m0 + wm * (TM * 16) + lr, rb = n0 + wn * (TN * 16) + lr;
#pragma unroll
        for (int j = 0; j < TN; j++) fb[0][j] = mm_tail(p.b, p.ldb, rb + j * 16, p.N, p.K, lp);
#pragma unroll
        for (int i = 0; i < TM; i++) fa[0][i] = mm_tail(p.a, p.lda, ra + i * 16, p.M, p.K, lp);
        mma(fa[0], fb[0]);
    }
    // Epilogue: 16 rows of the wave's outputs at a time through its own part of
    // LDS, so that rows leave in whole cache lines (a lane's four columns alone
    // are 32 bytes of a row per store instruction).
    constexpr int ES = (int)sizeof(TO), ROW = TN * 16 * ES, PITCH = ROW + 16, CH = ROW / 16;
    static_assert(16 * PITCH * NW <= ST * (SA + SB), "epilogue buffers");
    __syncthreads();                          // every wave is done with the stages
    int8_t* t = smem + wave * 16 * PITCH;     // a wave's LDS accesses keep their order
    TO* out = (TO*)p.out;
    const int64_t mw = m0 + wm * (TM * 16), nw = n0 + wn * (TN * 16);
    float sb[TN][4], bias[TN][4];
#pragma unroll
    for (int j = 0; j < TN && !kSplit; j++) {
        const int64_t n = nw + j * 16 + lp * 4;
#pragma unroll
        for (int r = 0; r < 4; r++) { sb[j][r] = 1.f; bias[j][r] = 0.f; }
        if (n + 4 <= p.N) {
            if (p.sb) __builtin_memcpy(sb[j], p.sb + n, 16);
            if (p.bias) __builtin_memcpy(bias[j], p.bias + n, 16);
        } else {
#pragma unroll
            for (int r = 0; r < 4; r++) {
                if (p.sb && n + r < p.N) sb[j][r] = p.sb[n + r];
                if (p.bias && n + r < p.N) bias[j][r] = p.bias[n + r];
            }
        }
    }
    float sa[TM];
#pragma unroll
    for (int i = 0; i < TM && !kSplit; i++) {
        const int64_t m = mw + i * 16 + lr;
        sa[i] = p.sa ? p.sa[m < p.M ? m : p.M - 1] : 1.f;
    }
#pragma unroll
    for (int i = 0; i < TM; i++) {
#pragma unroll
        for (int j = 0; j < TN; j++) {
            OutVec<TO> o;
#pragma unroll
            for (int r = 0; r < 4; r++) {
                if constexpr (kSplit) o.v[r] = acc[i][j][r];
                else o.v[r] = (TO)mm_out(acc[i][j][r], sa[i], sb[j][r], bias[j][r]);
            }
            *(OutVec<TO>*)(t + lr * PITCH + (j * 16 + lp * 4) * ES) = o;
        }
#pragma unroll
        for (int c = lane; c < 16 * CH; c += 64) {
            const int r = c / CH, q = c % CH;
            const v4i v = *(const v4i*)(t + r * PITCH + q * 16);
            const int64_t m = mw + i * 16 + r, n = nw + q * (16 / ES);
            if (m < p.M && n < p.N) {
                TO* d = out + m * p.ldc + n;
                if (n + 16 / ES <= p.N) {
                    __builtin_memcpy(d, &v, 16);
                } else {
                    TO e[16 / ES];
                    __builtin_memcpy(e, &v, 16);
#pragma unroll
                    for (int x = 0; x < 16 / ES; x++)
                        if (n + x < p.N) d[x] = e[x];
                }
            }
        }
    }
}

// Rows of a, of b or of both copied into buffers of zero-padded rows of Kp
// bytes (a multiple of 64): operands whose rows start off 16 bytes, where loads
// to LDS would straddle.  One pass over them, against M N K / 64 products (509 x
// 1001 x 1543 4.8 us beside 6.9 for the product).  Reading such rows into LDS
// through registers instead gains below 64 rows (33 x 1001 x 4097 12.9 to 9.6)
// and loses above (2048 x 2048 x 4095 33 to 72).
// pa, pb: NULL for an operand that stays.
__global__ __launch_bounds__(256) void k_mm_pack(MmArgs p, int8_t* __restrict__ pa, int8_t* __restrict__ pb, int64_t Kp)
{
    const int64_t pieces = Kp / 16, na = pa ? p.M * pieces : 0, all = na + (pb ? p.N * pieces : 0);
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const bool first = i < na;
        const int64_t e = first ? i : i - na, r = e / pieces, k = (e - r * pieces) * 16;
        const int8_t* row = first ? p.a + r * p.lda : p.b + r * p.ldb;
        *(v4i*)((first ? pa : pb) + r * Kp + k) = k > 0 && k + 20 <= p.K ? load16_odd(row, k) : load16(row, k, p.K);
    }
}

// Outputs from the int32 sums of `splits` (<= 16) parts of the reduction, four
// neighbours per thread; every part's load is in flight at once (64 x 2048 in 8
// parts 4.3 us).
template <typename TO>
__global__ __launch_bounds__(256) void k_mm_join(MmArgs p, const int32_t* __restrict__ part, int splits)
{
    const int64_t per = (p.N + 3) / 4;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < p.M * per; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, n = (i - m * per) * 4;
        const int32_t* q = part + m * p.ldc_part + n;
        v4i t[16];
#pragma unroll
        for (int k = 0; k < 16; k++) t[k] = *(const v4i*)(q + (k < splits ? k : 0) * p.M * p.ldc_part);
        v4i s = t[0];
#pragma unroll
        for (int k = 1; k < 16; k++)
            if (k < splits) s += t[k];
        const float sa = p.sa ? p.sa[m] : 1.f;
        OutVec<TO> o;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const bool in = n + r < p.N;
            o.v[r] = (TO)mm_out(s[r], sa, p.sb && in ? p.sb[n + r] : 1.f, p.bias && in ? p.bias[n + r] : 0.f);
        }
        TO* d = (TO*)p.out + m * p.ldc + n;
        if (n + 4 <= p.N) {
            __builtin_memcpy(d, &o, sizeof(o));
        } else {
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (n + r < p.N) d[r] = o.v[r];
        }
    }
}

// ---------------------------------------------------------------------------
// few rows of a: the bytes of b
// ---------------------------------------------------------------------------
// A block takes J * 16 rows of b, its NW waves deal out their reduction in
// pieces of 256; b comes straight into fragments (nothing of it is used
// twice), a from the caches, and the waves' sums meet in LDS.  Bound by b's
// bytes where N fills the CUs: 8 x 12288 x 4096 14.6 us from memory (3.4 TB/s),
// 12.4 from the last-level cache; 24 x 12288 x 4096 19.0 and 16.5.  The reduction
// is not split over blocks, so narrow outputs leave CUs idle: 8 x 1024 x 8192 8.2
// us (bytes 1.7), 8 x 256 x 16384 13.2 (0.9).
// ODD: rows of a or b may start off a multiple of four bytes.
template <typename TO, int MT, int J, int NW, bool ODD>
__global__ __launch_bounds__(NW * 64) void k_mm_rows(MmArgs p)
{
    __shared__ __attribute__((aligned(16))) int red[NW][MT * J][256];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int lr = lane & 15, lp = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (J * 16);
    const int8_t *ap[MT], *bp[J];
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int64_t r = i * 16 + lr;
        ap[i] = p.a + (r < p.M ? r : p.M - 1) * p.lda;
    }
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int64_t r = n0 + j * 16 + lr;
        bp[j] = p.b + (r < p.N ? r : p.N - 1) * p.ldb;
    }
    v4i acc[MT][J];
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < J; j++) acc[i][j] = (v4i){0, 0, 0, 0};
    const int K = (int)p.K;
    for (int k0 = w * 256; k0 < K; k0 += NW * 256) {
        v4i fa[4][MT], fb[4][J];
        if (ODD && k0 > 0 && k0 + 260 <= K) {
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int j = 0; j < J; j++) fb[u][j] = load16_odd(bp[j], k0 + u * 64 + lp * 16);
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int i = 0; i < MT; i++) fa[u][i] = load16_odd(ap[i], k0 + u * 64 + lp * 16);
        } else if (k0 + 256 <= K) {
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int j = 0; j < J; j++) __builtin_memcpy(&fb[u][j], bp[j] + k0 + u * 64 + lp * 16, 16);
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int i = 0; i < MT; i++) __builtin_memcpy(&fa[u][i], ap[i] + k0 + u * 64 + lp * 16, 16);
        } else {
#pragma unroll
            for (int u = 0; u < 4; u++) {
#pragma unroll
                for (int j = 0; j < J; j++) fb[u][j] = load16(bp[j], k0 + u * 64 + lp * 16, K);
#pragma unroll
                for (int i = 0; i < MT; i++) fa[u][i] = load16(ap[i], k0 + u * 64 + lp * 16, K);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
            for (int i = 0; i < MT; i++)
#pragma unroll
                for (int j = 0; j < J; j++)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][j], fa[u][i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < J; j++) *(v4i*)&red[w][i * J + j][lane * 4] = acc[i][j];
    __syncthreads();
    // output e of a 16 x 16 tile: row e / 16, column e % 16, held by lane
    // (e % 16) / 4 * 16 + e / 16 in element e % 4
    for (int e = tid; e < MT * J * 256; e += NW * 64) {
        const int col = e % (J * 16), row = e / (J * 16);
        const int64_t n = n0 + col;
        if (row >= p.M || n >= p.N) continue;
        const int t = (row >> 4) * J + (col >> 4), r = row & 15, c = col & 15;
        const int at = ((c >> 2) * 16 + r) * 4 + (c & 3);
        int sum = 0;
#pragma unroll
        for (int i = 0; i < NW; i++) sum += red[i][t][at];
        ((TO*)p.out)[row * p.ldc + n] =
            (TO)mm_out(sum, p.sa ? p.sa[row] : 1.f, p.sb ? p.sb[n] : 1.f, p.bias ? p.bias[n] : 0.f);
    }
}

// ---------------------------------------------------------------------------
// one token of a whole linear layer
// ---------------------------------------------------------------------------
struct LinArgs {
    MmArgs p;                    // a: unused
    const void* x;
    int8_t* codes;
    float* scale;
    int32_t bits, mode;
    int32_t* status;
};

constexpr int kTokenMax = 8192;            // longest token that a block quantizes for itself

// k_mm_rows for one token, whose blocks quantize it for themselves: the first
// weights are on their way while a block takes the maximum and leaves the
// codes in LDS.  x is read by every block, from the caches; of the codes each
// block writes out its own share.  1 x 4096 x 4096 6.7 us with weights from
// memory (2.5 TB/s), 5.3 from the caches: load, maximum, codes, products and sum
// follow one another, and only each wave's first 256 of the reduction are
// requested ahead of the maximum, the others piece by piece behind the codes.
template <typename TX, typename TO, int J>
__global__ __launch_bounds__(512) void k_linear_token(LinArgs a)
{
    constexpr int NW = 8, N = RowVec<TX>::N, VPT = kTokenMax / N / 512;
    __shared__ __attribute__((aligned(16))) int red[NW][J][16];
    __shared__ uint32_t top[NW];
    __shared__ __attribute__((aligned(16))) int8_t cd[kTokenMax];
    const MmArgs& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int lr = lane & 15, lp = lane >> 4;
    const int K = (int)p.K, Kp = (K + 255) & ~255;
    const int64_t n0 = (int64_t)blockIdx.x * (J * 16);
    const TX* x = (const TX*)a.x;
    RowSlot<N> sl[VPT];
    RowVec<TX> xv[VPT];
#pragma unroll
    for (int j = 0; j < VPT; j++) {
        sl[j] = row_slot<N>(((int64_t)j * 512 + tid) * N, K);
        xv[j] = slot_load<TX, N>(x, sl[j]);
    }
    const int8_t* bp[J];
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int64_t r = n0 + j * 16 + lr;
        bp[j] = p.b + (r < p.N ? r : p.N - 1) * p.ldb;
    }
    v4i fb[4][J];
    auto weights = [&](int k0) {
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
            for (int j = 0; j < J; j++) {
                const int k = k0 + u * 64 + lp * 16;
                if (k0 + 256 <= K) __builtin_memcpy(&fb[u][j], bp[j] + k, 16);
                else fb[u][j] = load16(bp[j], k, K);
            }
    };
    if (w * 256 < K) weights(w * 256);
    uint32_t big = 0;
#pragma unroll
    for (int j = 0; j < VPT; j++)
#pragma unroll
        for (int i = 0; i < N; i++) {
            const uint32_t b = bits_of((float)xv[j].v[i]);
            big = b > big ? b : big;
        }
    big = wave_top_u32(big);
    if (lane == 0) top[w] = big;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; i++) big = top[i] > big ? top[i] : big;
    const float s = scale_of(bits_of((double)__builtin_bit_cast(float, big)), a.bits, a.mode);
    const Coder k(s);
    const int lim = (1 << (a.bits - 1)) - 1;
    if (blockIdx.x == 0 && tid == 0) {
        *a.scale = s;
        if (!k.ok) set_status(a.status, ISEG_DEV_NONFINITE);
    }
#pragma unroll
    for (int j = 0; j < VPT; j++)
        if (sl[j].dup < N) {
            float f[N];
#pragma unroll
            for (int i = 0; i < N; i++) f[i] = (float)xv[j].v[i];
            uint32_t o[N / 4];
            codes_of<N, false>(f, f, [&](int) -> const Coder& { return k; }, lim, o);
            __builtin_memcpy(cd + sl[j].at, o, N);
        }
    if (tid < Kp - K) cd[K + tid] = 0;
    __syncthreads();
    // this block's share of the codes
    for (int64_t q = ((int64_t)blockIdx.x * 512 + tid) * 16; q < K; q += (int64_t)gridDim.x * 512 * 16) {
        if (q + 16 <= K) *(v4i*)(a.codes + q) = *(const v4i*)(cd + q);
        else
            for (int64_t e = q; e < K; e++) a.codes[e] = cd[e];
    }
    v4i acc[J];
#pragma unroll
    for (int j = 0; j < J; j++) acc[j] = (v4i){0, 0, 0, 0};
    for (int k0 = w * 256; k0 < K; k0 += NW * 256) {
        if (k0 != w * 256) weights(k0);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const v4i fa = *(const v4i*)(cd + k0 + u * 64 + lp * 16);      // the token in all 16 rows
#pragma unroll
            for (int j = 0; j < J; j++)
                acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][j], fa, acc[j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < J; j++)
        if (lr == 0) *(v4i*)&red[w][j][lp * 4] = acc[j];
    __syncthreads();
    if (tid < J * 16 && n0 + tid < p.N) {
        const int64_t n = n0 + tid;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < NW; i++) sum += red[i][tid >> 4][tid & 15];
        ((TO*)p.out)[n] = (TO)mm_out(sum, s, p.sb ? p.sb[n] : 1.f, p.bias ? p.bias[n] : 0.f);
    }
}

constexpr int kMmThreads = 512;            // of every product kernel's block
constexpr int64_t kMmBlocks = ((int64_t)1 << 32) / kMmThreads - 1;      // a launch's threads fit 32 bits

template <typename TO, int BM, int BN, int WM, int WN, int ST>
int launch_tile(MmArgs p, hipStream_t s, int splits = 1)
{
    constexpr size_t lds = (size_t)ST * (BM + BN) * 128;
    static_assert(WM * WN * 64 == kMmThreads, "what mm_plan counts with");
    if (lds > 65536 && !lds_limit((const void*)k_mm_tile<TO, BM, BN, WM, WN, ST>, lds)) return ISEG_ERR_DEVICE;
    p.tm = (uint32_t)ceil_div64(p.M, BM);
    p.tn = (uint32_t)ceil_div64(p.N, BN);
    hipLaunchKernelGGL((k_mm_tile<TO, BM, BN, WM, WN, ST>), dim3(p.tm * p.tn, splits), dim3(WM * WN * 64), lds, s, p);
    return launch_ok();
}

template <typename TO, int MT, int J, int NW>
int launch_rows(const MmArgs& p, hipStream_t s)
{
    static_assert(NW * 64 == kMmThreads, "what mm_check counts with");
    const int64_t nb = ceil_div64(p.N, J * 16);
    if (((uintptr_t)p.a | (uintptr_t)p.b | (uintptr_t)p.lda | (uintptr_t)p.ldb) & 3)
        hipLaunchKernelGGL((k_mm_rows<TO, MT, J, NW, true>), dim3((unsigned)nb), dim3(NW * 64), 0, s, p);
    else
        hipLaunchKernelGGL((k_mm_rows<TO, MT, J, NW, false>), dim3((unsigned)nb), dim3(NW * 64), 0, s, p);
    return launch_ok();
}

template <typename TO, int BM, int BN, int WM, int WN, int ST>
int launch_split(const MmArgs& p, int splits, int32_t* ws, hipStream_t s)
{
    MmArgs q = p;
    q.ksplit = ceil_div64(ceil_div64(p.K, 128), splits) * 128;
    q.out = ws;
    q.ldc = q.ldc_part = (p.N + 3) / 4 * 4;
    const int n = (int)ceil_div64(p.K, q.ksplit);
    const int rc = launch_tile<int32_t, BM, BN, WM, WN, ST>(q, s, n);
    if (rc != ISEG_OK) return rc;
    MmArgs r = p;
    r.ldc_part = q.ldc_part;
    hipLaunchKernelGGL(k_mm_join<TO>, dim3(grid_for(p.M * (q.ldc_part / 4), 256, 1 << 16)), dim3(256), 0, s, r,
                       (const int32_t*)ws, n);
    return launch_ok();
}

// How a product is run.  The tile kernels' times on MI355X, in us without the
// launch, for one round of blocks over the 256 CUs (te + ts per 128 of the
// reduction), once with one block per CU and once with as many as fit:
//   256 x 256           9.7 + 1.55        (one fits)
//   192 x 192           6.0 + 1.13        (one fits)
//   128 x 192           4.5 + 0.8         5.5 + 1.27
//   128 x 128           3.5 + 0.6 (four stages)   4.2 + 0.9 (two blocks of two stages)
//   64 x 128            2.0 + 0.3         3.0 + 0.7
//   64 x 64             0.6 + 0.27        1.5 + 0.55
// The plan with the least estimate is taken; a reduction cut into parts costs
// a second kernel (4.5 us).  Measured beside it: 2048 x 8192 x 2048, 256 tiles
// of 256 x 256 39.0 us, 128 x 128 44.8; 4544 x 1824 x 7488, 240 tiles of 192 x
// 192 76, 144 of 256 x 256 102; 1024 x 2048 x 2048, 64 x 128 9.4, 128 x 128
// 12.7; 64 x 2048 x 8192, 64 x 64 in 8 parts 12.3, in one 20.7.
enum MmKind { MM_ROWS16, MM_ROWS32, MM_256, MM_192, MM_128x192, MM_128, MM_128_DEEP, MM_64x128, MM_64 };
struct MmPlan {
    MmKind kind;
    int splits;
    bool pack_a, pack_b;         // may have to be packed
};

MmPlan mm_plan(const iseg_matmul_geom* g)
{
    // few rows: b's bytes are what counts (see k_mm_rows)
    if (g->M <= 32) return {g->M <= 16 ? MM_ROWS16 : MM_ROWS32, 1, false, false};
    struct Kind {
        MmKind one, full;
        int64_t bm, bn;
        int fit;
        double te1, ts1, te, ts;
    };
    static const Kind kinds[] = {
        {MM_256, MM_256, 256, 256, 1, 9.7, 1.55, 9.7, 1.55},
        {MM_192, MM_192, 192, 192, 1, 6.0, 1.13, 6.0, 1.13},
        {MM_128x192, MM_128x192, 128, 192, 2, 4.5, 0.8, 5.5, 1.27},
        {MM_128_DEEP, MM_128, 128, 128, 2, 3.5, 0.6, 4.2, 0.9},
        {MM_64x128, MM_64x128, 64, 128, 2, 2.0, 0.3, 3.0, 0.7},
        {MM_64, MM_64, 64, 64, 2, 0.6, 0.27, 1.5, 0.55},
    };
    const int64_t st = ceil_div64(g->K, 128);
    MmPlan best = {MM_64, 1, false, false};
    double least = 1e30;
    for (const Kind& k : kinds) {
        const int64_t tiles = ceil_div64(g->M, k.bm) * ceil_div64(g->N, k.bn);
        if (tiles > kMmBlocks) continue;
        const double t = tiles <= 256 ? k.te1 + k.ts1 * (double)st
                                      : (double)ceil_div64(tiles, 256 * k.fit) * (k.te + k.ts * (double)st);
        if (t < least) { least = t; best = {tiles <= 256 ? k.one : k.full, 1, false, false}; }
        if (k.one == MM_64 && tiles <= 128) {
            int64_t sp = 256 / tiles < 16 ? 256 / tiles : 16;
            sp = sp < st / 4 ? sp : st / 4;              // parts of at least 512 of the reduction
            const double u = sp > 1 ? k.te1 + k.ts1 * (double)ceil_div64(st, sp) + 4.5 : 1e30;
            if (u < least) { least = u; best = {MM_64, (int)sp, false, false}; }
        }
    }
    best.pack_a = g->unaligned || g->lda % 16;
    best.pack_b = g->unaligned || g->ldb % 16;
    return best;
}

int64_t mm_packed_row(int64_t K) { return (K + 63) / 64 * 64; }

size_t mm_pack_bytes(const iseg_matmul_geom* g, const MmPlan& pl)
{
    const size_t Kp = (size_t)mm_packed_row(g->K);
    return (pl.pack_a ? align256((size_t)g->M * Kp) : 0) + (pl.pack_b ? align256((size_t)g->N * Kp) : 0);
}

template <typename TO>
int launch_mm(MmArgs p, const iseg_matmul_geom* g, const MmPlan& pl, char* ws, hipStream_t s)
{
    // Rows of b per block and waves on them, 16-row products on 1 x 4096 x 4096
    // / 8 x 12288 x 4096: 16 rows, 8 waves 6.5 / 17.0 us, 32 rows 7.0 / 14.1.
    if (pl.kind == MM_ROWS16) return g->N <= 8192 ? launch_rows<TO, 1, 1, 8>(p, s) : launch_rows<TO, 1, 2, 8>(p, s);
    if (pl.kind == MM_ROWS32) return g->N <= 4096 ? launch_rows<TO, 2, 1, 8>(p, s) : launch_rows<TO, 2, 2, 8>(p, s);
    if (p.K > 0) {
        const int64_t Kp = mm_packed_row(p.K);
        int8_t* pa = pl.pack_a && ((p.lda | (int64_t)(uintptr_t)p.a) & 15) ? (int8_t*)ws : nullptr;
        int8_t* pb = pl.pack_b && ((p.ldb | (int64_t)(uintptr_t)p.b) & 15)
                         ? (int8_t*)ws + (pl.pack_a ? align256((size_t)p.M * Kp) : 0) : nullptr;
        if (pa || pb) {
            const int64_t rows = (pa ? p.M : 0) + (pb ? p.N : 0);
            hipLaunchKernelGGL(k_mm_pack, dim3(grid_for(rows * (Kp / 16), 256, 8192)), dim3(256), 0, s, p, pa, pb, Kp);
            if (pa) { p.a = pa; p.lda = Kp; }
            if (pb) { p.b = pb; p.ldb = Kp; }
            if (pa && pb) p.K = Kp;           // both padded with zeros: no broken last piece
        }
    }
    switch (pl.kind) {
    case MM_256: return launch_tile<TO, 256, 256, 2, 4, 2>(p, s);
    case MM_192: return launch_tile<TO, 192, 192, 2, 4, 3>(p, s);
    case MM_128x192: return launch_tile<TO, 128, 192, 2, 4, 2>(p, s);
    case MM_128: return launch_tile<TO, 128, 128, 2, 4, 2>(p, s);
    case MM_128_DEEP: return launch_tile<TO, 128, 128, 2, 4, 4>(p, s);
    case MM_64x128: return launch_tile<TO, 64, 128, 2, 4, 3>(p, s);
    default:
        if (pl.splits > 1) return launch_split<TO, 64, 64, 2, 4, 4>(p, pl.splits, (int32_t*)(ws + mm_pack_bytes(g, pl)), s);
        return launch_tile<TO, 64, 64, 2, 4, 4>(p, s);
    }
}

int mm_check(const iseg_matmul_geom* g)
{
    if (!g || !is_float_dtype(g->out_dtype)) return ISEG_ERR_ARG;
    const int64_t big = (int64_t)1 << 31;
    if (g->M < 0 || g->N < 0 || g->K < 0 || g->M >= big || g->N >= big || g->lda < g->K || g->ldb < g->K ||
        g->ldc < g->N)
        return ISEG_ERR_SHAPE;
    if (g->K > 131071) return ISEG_ERR_UNSUPPORTED;
    // one launch: 32 rows of b per block, or the largest tiles
    const int64_t blocks = g->M <= 32 ? (g->M > 0 ? ceil_div64(g->N, 32) : 0)
                                      : ceil_div64(g->M, 256) * ceil_div64(g->N, 256);
    return blocks <= kMmBlocks ? ISEG_OK : ISEG_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" size_t iseg_matmul_i8_ws(const iseg_matmul_geom* g)
{
    if (mm_check(g) != ISEG_OK) return 0;
    if (g->M == 0 || g->N == 0) return kNoWs;
    const MmPlan pl = mm_plan(g);
    size_t b = mm_pack_bytes(g, pl);
    if (pl.splits > 1) b += align256((size_t)pl.splits * g->M * ((g->N + 3) / 4 * 4) * 4);
    return b ? ws_used(b) : kNoWs;
}

extern "C" int iseg_matmul_i8(const int8_t* a, const float* a_scale, const int8_t* b, const float* b_scale,
                              const float* bias, const iseg_matmul_geom* g, void* out, void* ws, size_t ws_bytes,
                              hipStream_t stream)
{
    const int rc = mm_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->M == 0 || g->N == 0) return ISEG_OK;
    if (!out || (g->K > 0 && (!a || !b))) return ISEG_ERR_ARG;
    if (!g->unaligned && (((uintptr_t)a | (uintptr_t)b) & 15)) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_matmul_i8_ws(g)) return ISEG_ERR_WORKSPACE;
    MmArgs p = {};
    p.a = a; p.b = b; p.sa = a_scale; p.sb = b_scale; p.bias = bias; p.out = out;
    p.M = g->M; p.N = g->N; p.K = g->K; p.lda = g->lda; p.ldb = g->ldb; p.ldc = g->ldc;
    const MmPlan pl = mm_plan(g);
    return g->out_dtype == ISEG_F32   ? launch_mm<float>(p, g, pl, (char*)ws, stream)
           : g->out_dtype == ISEG_F16 ? launch_mm<f16_t>(p, g, pl, (char*)ws, stream)
                                      : launch_mm<bf16_t>(p, g, pl, (char*)ws, stream);
}

// ---------------------------------------------------------------------------
// linear layer
// ---------------------------------------------------------------------------
namespace {

iseg_matmul_geom lin_product(const iseg_linear_geom* g)
{
    return {g->M, g->N, g->K, g->codes_ld, g->w_ld, g->y_ld, g->y_dtype, g->unaligned};
}

int lin_check(const iseg_linear_geom* g)
{
    if (!g || !is_float_dtype(g->x_dtype) || !is_float_dtype(g->y_dtype) || g->bits < 2 || g->bits > 8 ||
        (g->scale_mode != ISEG_SCALE_MAX && g->scale_mode != ISEG_SCALE_POW2) || g->reserved)
        return ISEG_ERR_ARG;
    if (g->x_ld < g->K || g->codes_ld % 16) return ISEG_ERR_SHAPE;
    const iseg_matmul_geom p = lin_product(g);
    return mm_check(&p);
}

// One kernel for one token, at every size that a block can hold: N x K 1024 x
// 1024 3.2 us against 5.4 for the two, 4096 x 4096 6.7 / 9.1 (from the caches 5.3 /
// 7.4), 1024 x 8192 8.0 / 10.3, 4096 x 8192 10.3 / 12.0, 12288 x 4096 16.2 / 17.1,
// 8192 x 8192 15.7 / 18.8.  What it saves is a launch, the more of the whole the
// fewer the weights' bytes.  (With more tokens every block's own quantization
// costs more than the launch: two tokens of 4096 10.5 us against 9.3.)
bool lin_fused(const iseg_linear_geom* g)
{
    return g->M == 1 && g->N > 0 && g->K >= 8 && g->K <= kTokenMax;
}

template <typename TX, typename TO>
int launch_linear(const LinArgs& a, hipStream_t s)
{
    const bool two = a.p.N > 8192;         // rows of b per block as for k_mm_rows
    const int64_t nb = ceil_div64(a.p.N, two ? 32 : 16);
    if (two) hipLaunchKernelGGL((k_linear_token<TX, TO, 2>), dim3((unsigned)nb), dim3(512), 0, s, a);
    else hipLaunchKernelGGL((k_linear_token<TX, TO, 1>), dim3((unsigned)nb), dim3(512), 0, s, a);
    return launch_ok();
}

template <typename TX>
int launch_linear_out(const LinArgs& a, int32_t t, hipStream_t s)
{
    return t == ISEG_F32 ? launch_linear<TX, float>(a, s)
                         : t == ISEG_F16 ? launch_linear<TX, f16_t>(a, s) : launch_linear<TX, bf16_t>(a, s);
}

}  // namespace

extern "C" size_t iseg_linear_i8_fwd_ws(const iseg_linear_geom* g)
{
    if (lin_check(g) != ISEG_OK) return 0;
    const iseg_matmul_geom p = lin_product(g);
    return lin_fused(g) ? kNoWs : iseg_matmul_i8_ws(&p);
}

extern "C" int iseg_linear_i8_fwd(const void* x, const int8_t* w, const float* w_scale, const float* bias,
                                  const iseg_linear_geom* g, int8_t* codes, float* scale, void* y, void* ws,
                                  size_t ws_bytes, int32_t* dev_status, hipStream_t stream)
{
    int rc = lin_check(g);
    if (rc != ISEG_OK) return rc;
    if (g->M == 0) return ISEG_OK;
    if (!scale || (g->K > 0 && (!x || !codes)) || (g->N > 0 && (!y || (g->K > 0 && !w)))) return ISEG_ERR_ARG;
    if (((uintptr_t)codes & 15) || (!g->unaligned && ((uintptr_t)w & 15))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_linear_i8_fwd_ws(g)) return ISEG_ERR_WORKSPACE;
    if (lin_fused(g)) {
        LinArgs a = {};
        a.p.b = w; a.p.sb = w_scale; a.p.bias = bias; a.p.out = y;
        a.p.M = g->M; a.p.N = g->N; a.p.K = g->K; a.p.ldb = g->w_ld; a.p.ldc = g->y_ld;
        a.x = x; a.codes = codes; a.scale = scale;
        a.bits = g->bits; a.mode = g->scale_mode; a.status = dev_status;
        return g->x_dtype == ISEG_F32   ? launch_linear_out<float>(a, g->y_dtype, stream)
               : g->x_dtype == ISEG_F16 ? launch_linear_out<f16_t>(a, g->y_dtype, stream)
                                        : launch_linear_out<bf16_t>(a, g->y_dtype, stream);
    }
    rc = iseg_quantize_rows(x, g->x_dtype, g->M, g->K, g->x_ld, nullptr, g->bits, g->scale_mode, codes, g->codes_ld,
                            scale, dev_status, stream);
    if (rc != ISEG_OK) return rc;
    const iseg_matmul_geom p = lin_product(g);
    return iseg_matmul_i8(codes, scale, w, w_scale, bias, &p, y, ws, ws_bytes, stream);
}

// ---------------------------------------------------------------------------
// backward of the linear layer
// ---------------------------------------------------------------------------
namespace {

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

int lbw_check(const iseg_linear_bwd_geom* g)
{
    if (!g || !is_float_dtype(g->dy_dtype) || !is_float_dtype(g->out_dtype) || g->bits < 2 || g->bits > 8 ||
        (g->scale_mode != ISEG_SCALE_MAX && g->scale_mode != ISEG_SCALE_POW2) || g->reserved)
        return ISEG_ERR_ARG;
    const int64_t big = (int64_t)1 << 31;
    if (g->M < 0 || g->N < 0 || g->K < 0 || g->M >= big || g->N >= big || g->K >= big || g->dy_ld < g->N ||
        g->a_ld < g->K || g->w_ld < g->K || (g->wt_ld && g->wt_ld < g->N) || g->dx_ld < g->K || g->dw_ld < g->K)
        return ISEG_ERR_SHAPE;
    return ISEG_OK;
}

// products of the two gradients: dx = Q_rows(dy) [M, N] x w^T, dw = Q_cols(dy) [N, M] x a^T
iseg_matmul_geom lbw_dx(const iseg_linear_bwd_geom* g)
{
    return {g->M, g->K, g->N, up16(g->N), g->wt_ld ? g->wt_ld : up16(g->N), g->dx_ld, g->out_dtype, g->unaligned};
}

iseg_matmul_geom lbw_dw(const iseg_linear_bwd_geom* g)
{
    return {g->N, g->K, g->M, up16(g->M), up16(g->M), g->dw_ld, g->out_dtype, 0};
}

// The workspace, the same for both gradients, which run one after the other:
// codes, scales, the transposed second operand, the quantizer's own, the product's own.
struct LbwWs {
    size_t codes, scale, turned, quant, product, total;
};

LbwWs lbw_ws(const iseg_linear_bwd_geom* g, bool dw)
{
    const iseg_matmul_geom p = dw ? lbw_dw(g) : lbw_dx(g);
    LbwWs w = {};
    w.codes = 0;
    w.scale = align256((size_t)p.M * p.lda);
    w.turned = w.scale + align256((size_t)p.M * 4);
    w.quant = w.turned + (dw || !g->wt_ld ? align256((size_t)p.N * p.ldb) : 0);
    w.product = w.quant + (dw ? align256(iseg_quantize_cols_ws(g->M, g->N)) : 0);
    w.total = w.product + iseg_matmul_i8_ws(&p);
    return w;
}

}  // namespace

extern "C" size_t iseg_linear_i8_bwd_ws(const iseg_linear_bwd_geom* g)
{
    if (lbw_check(g) != ISEG_OK) return 0;
    const size_t a = lbw_ws(g, false).total, b = lbw_ws(g, true).total;
    return ws_used(a > b ? a : b);
}

extern "C" int iseg_linear_i8_bwd(const void* dy, const int8_t* a, const float* a_scale, const int8_t* w,
                                  const float* w_scale, const int8_t* w_t, const iseg_linear_bwd_geom* g, void* dx,
                                  void* dw, float* dbias, void* ws, size_t ws_bytes, int32_t* dev_status,
                                  hipStream_t stream)
{
    int rc = lbw_check(g);
    if (rc != ISEG_OK) return rc;
    // what is asked for, of what is not empty
    const bool want_x = dx && g->M > 0 && g->K > 0, want_w = dw && g->N > 0 && g->K > 0, want_b = dbias && g->N > 0;
    const iseg_matmul_geom px = lbw_dx(g), pw = lbw_dw(g);
    if ((want_x && (rc = mm_check(&px)) != ISEG_OK) || (want_w && (rc = mm_check(&pw)) != ISEG_OK)) return rc;
    if (((want_w || want_b) && g->N > kMaxTurned) || ((want_w || (want_x && !g->wt_ld)) && g->K > kMaxTurned))
        return ISEG_ERR_UNSUPPORTED;
    if (g->M > 0 && g->N > 0 && (want_x || want_w || want_b) && !dy) return ISEG_ERR_ARG;
    if (want_x && g->N > 0 && !(g->wt_ld ? w_t : w)) return ISEG_ERR_ARG;
    if (want_x && g->wt_ld && !g->unaligned && ((uintptr_t)w_t & 15)) return ISEG_ERR_ARG;
    if (want_w && g->M > 0 && !a) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_linear_i8_bwd_ws(g)) return ISEG_ERR_WORKSPACE;
    char* base = (char*)ws;
    if (want_x) {
        const iseg_matmul_geom& p = px;
        const LbwWs o = lbw_ws(g, false);
        int8_t* codes = (int8_t*)(base + o.codes);
        float* scale = (float*)(base + o.scale);
        const int8_t* wt = w_t;
        if (!g->wt_ld) {
            rc = iseg_transpose_i8(w, g->N, g->K, g->w_ld, (int8_t*)(base + o.turned), p.ldb, stream);
            if (rc != ISEG_OK) return rc;
            wt = (const int8_t*)(base + o.turned);
        }
        rc = iseg_quantize_rows(dy, g->dy_dtype, g->M, g->N, g->dy_ld, w_scale, g->bits, g->scale_mode, codes, p.lda,
                                scale, dev_status, stream);
        if (rc != ISEG_OK) return rc;
        rc = iseg_matmul_i8(codes, scale, wt, nullptr, nullptr, &p, dx, base + o.product, ws_bytes - o.product, stream);
        if (rc != ISEG_OK) return rc;
    }
    if (want_w || want_b) {
        const iseg_matmul_geom& p = pw;
        const LbwWs o = lbw_ws(g, true);
        int8_t* codes = (int8_t*)(base + o.codes);
        float* scale = (float*)(base + o.scale);
        int8_t* at = (int8_t*)(base + o.turned);
        const TurnJob job = {a, g->M, g->K, g->a_ld, at, p.ldb};
        rc = quantize_cols_turn(dy, g->dy_dtype, g->M, g->N, g->dy_ld, a_scale, g->bits, g->scale_mode, codes, p.lda,
                                scale, dbias, base + o.quant, o.product - o.quant, dev_status, want_w ? &job : nullptr,
                                stream);
        if (rc != ISEG_OK) return rc;
        if (want_w) {
            rc = iseg_matmul_i8(codes, scale, at, nullptr, nullptr, &p, dw, base + o.product, ws_bytes - o.product,
                                stream);
        }
    }
    return rc;
}
