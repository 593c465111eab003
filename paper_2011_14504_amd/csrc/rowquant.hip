// rowquant.hip -- quantizers with a scale for each row or each column, and the
// transposition of int8 codes: the operands of iseg_matmul_i8.
//
// The decisions are exact (coder.h).
#include "coder.h"

namespace {

struct RqRowArgs {
    const void* x;
    const float* mul;
    int8_t* codes;
    float *scale, *sums;
    uint64_t* pmax;              // columns: [strips][C] bit patterns of the largest |v|
    float* psum;                 // columns: [strips][C] partial sums of x
    int64_t M, C, x_ld, codes_ld;
    int32_t bits, mode;
    int32_t* status;
};

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
// largest bit pattern over the NW waves of a row (red: NW words that no
// earlier call may still read)
template <int NW>
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v, uint32_t* red)
{
    v = wave_top_u32(v);
    if (NW == 1) return v;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (lane == 0) red[w] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < NW; i++) v = red[i] > v ? red[i] : v;
    return v;
}

// NW waves per row (one, or the whole block), VPT vectors of it per thread, in
// registers between the maximum and the codes, and the next row's on their way.
// x is read and the codes written once: 4096 x 4096 bf16 14.6 us (3.4 TB/s), fp32
// 16.3 (5.1), 4096 x 16384 bf16 41.5 (4.9).  fp32 is bound by memory, 16-bit types
// as much by the issue of 24 vector instructions per element (40 of 43 us at
// 16384 x 4096, by counters).  mul waits in LDS,
// every thread's own part: in registers as well it leaves one block of eight
// waves on a CU (4096 x 16384 bf16 81 us, so 54 at four waves per SIMD).
template <typename T, bool MUL, int NW, int VPT>
__global__ __launch_bounds__(NW < 4 ? 256 : NW * 64) __attribute__((amdgpu_waves_per_eu(NW == 8 ? 4 : 1))) void
k_quantize_rows(RqRowArgs a)
{
    constexpr int N = RowVec<T>::N;
    constexpr int NT = NW * 64, R = NW < 4 ? 4 / NW : 1;
    __shared__ uint32_t red[2][NW];
    __shared__ unsigned long long top[2];
    extern __shared__ __attribute__((aligned(16))) float4 ms[];        // MUL: [VPT * N / 4][threads of the block]
    const int tid = threadIdx.x % NT;
    RowSlot<N> sl[VPT];                                       // only the last one may be short
#pragma unroll
    for (int j = 0; j < VPT; j++) {
        const int64_t c = ((int64_t)j * NT + tid) * N;
        sl[j] = j < VPT - 1 ? RowSlot<N>{c, 0} : row_slot<N>(c, a.C);
        if (MUL) {
            const ParamVec<float, N> mv = param_load<float, N>(a.mul, sl[j], 0.f);
#pragma unroll
            for (int q = 0; q < N / 4; q++) __builtin_memcpy(&ms[(j * (N / 4) + q) * (R * NT) + threadIdx.x], mv.v + q * 4, 16);
        }
    }
    auto mul_of = [&](int j) {
        ParamVec<float, N> mv = {};
#pragma unroll
        for (int q = 0; q < N / 4 && MUL; q++) __builtin_memcpy(mv.v + q * 4, &ms[(j * (N / 4) + q) * (R * NT) + threadIdx.x], 16);
        return mv;
    };
    const int lim = (1 << (a.bits - 1)) - 1;
    RowVec<T> nv[VPT];
    int64_t m = (int64_t)blockIdx.x * R + threadIdx.x / NT;
    const int64_t step = (int64_t)gridDim.x * R;
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < VPT; j++) nv[j] = slot_load<T, N>((const T*)a.x + r * a.x_ld, sl[j]);
    };
    if (m < a.M) fetch(m);
    int flip = 0;
    for (; m < a.M; m += step, flip ^= 1) {
        RowVec<T> xv[VPT];
        uint32_t big = 0;
#pragma unroll
        for (int j = 0; j < VPT; j++) xv[j] = nv[j];
        if (m + step < a.M) fetch(m + step);
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const ParamVec<float, N> mv = mul_of(j);
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float x = (float)xv[j].v[i];
                const uint32_t b = bits_of(MUL ? x * mv.v[i] : x);
                big = b > big ? b : big;
            }
        }
        const uint32_t mine = big;
        big = row_max_u32<NW>(big, red[flip]);
        uint64_t tb;
        if constexpr (MUL) {
            // The exact products of the elements that reach the float maximum, in
            // the few threads that have one: big + l, l = |x mul| - big exact by
            // one fma.  Where that may be subnormal, or big is infinite, they are
            // read again and formed in double.
            uint64_t e = 0;
            if (mine == big) {
                const float fb = __builtin_bit_cast(float, big);
                float l = -__builtin_inff();
                uint32_t any = 0;
#pragma unroll
                for (int j = 0; j < VPT; j++) {
                    const ParamVec<float, N> mv = mul_of(j);
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        const float x = (float)xv[j].v[i];
                        any |= bits_of(x);
                        if (bits_of(x * mv.v[i]) == big) l = fmaxf(l, fmaf(fabsf(x), fabsf(mv.v[i]), -fb));
                    }
                }
                if (fb >= 8.6736174e-19f && fb <= 3.4028234e38f) {
                    e = bits_of((double)fb + (double)l);
                } else if (any | big) {
                    const T* x = (const T*)a.x + m * a.x_ld;
                    for (int j = 0; j < VPT; j++)
                        for (int64_t c = ((int64_t)j * NT + tid) * N; c < ((int64_t)j * NT + tid + 1) * N && c < a.C; c++) {
                            const float f = (float)x[c];
                            const uint64_t b = bits_of((double)f * (double)a.mul[c]);
                            if (bits_of(f * a.mul[c]) == big && b > e) e = b;
                        }
                }
            }
            if (NW == 1) {
                tb = wave_max_u64(e);
            } else {
                if (threadIdx.x == 0) top[flip] = 0;
                __syncthreads();
                if (e) atomicMax(&top[flip], (unsigned long long)e);
                __syncthreads();
                tb = top[flip];
            }
        } else {
            tb = bits_of((double)__builtin_bit_cast(float, big));
        }
        const float s = scale_of(tb, a.bits, a.mode);
        const Coder k(s);
        if (tid == 0) {
            a.scale[m] = s;
            if (!k.ok) set_status(a.status, ISEG_DEV_NONFINITE);
        }
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            float x[N];
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = (float)xv[j].v[i];
            uint32_t o[N / 4];
            const ParamVec<float, N> mv = mul_of(j);
            codes_of<N, MUL>(x, mv.v, [&](int) -> const Coder& { return k; }, lim, o);
            if (j < VPT - 1 || sl[j].dup < N) __builtin_memcpy(a.codes + m * a.codes_ld + sl[j].at, o, N);
        }
    }
}

// rows longer than the registers take: read twice, the second time from the
// caches (4096 x 50000 bf16 203 us, 3.0 TB/s of x and codes)
template <typename T, bool MUL>
__global__ __launch_bounds__(1024) void k_quantize_rows_long(RqRowArgs a)
{
    constexpr int N = RowVec<T>::N, U = 2;
    const int lim = (1 << (a.bits - 1)) - 1;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* x = (const T*)a.x + m * a.x_ld;
        uint64_t e = 0;
        uint32_t big = 0;
        for (int64_t c = threadIdx.x * N; c < a.C; c += U * 1024 * N) {
            RowVec<T> v[U];
            ParamVec<float, N> mv[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const RowSlot<N> sl = row_slot<N>(c + u * 1024 * N, a.C);
                v[u] = slot_load<T, N>(x, sl);                // zeros without a vector
                if (MUL) mv[u] = param_load<float, N>(a.mul, sl, 0.f);
            }
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const float f = (float)v[u].v[i];
                    const uint32_t b = bits_of(MUL ? f * mv[u].v[i] : f);
                    if (MUL) {
                        // the exact product, of what reaches the largest so far
                        if (b >= big) {
                            const uint64_t t = bits_of((double)f * (double)mv[u].v[i]);
                            e = t > e ? t : e;
                        }
                    }
                    big = b > big ? b : big;
                }
        }
        if (!MUL) e = bits_of((double)__builtin_bit_cast(float, big));
        const float s = scale_of(block_max_u64(e), a.bits, a.mode);
        const Coder k(s);
        if (threadIdx.x == 0) {
            a.scale[m] = s;
            if (!k.ok) set_status(a.status, ISEG_DEV_NONFINITE);
        }
        int8_t* o = a.codes + m * a.codes_ld;
        for (int64_t c = threadIdx.x * N; c < a.C; c += 1024 * N) {
            const RowSlot<N> sl = row_slot<N>(c, a.C);
            const RowVec<T> v = row_load(x + sl.at);
            ParamVec<float, N> mv;
            if (MUL) mv = param_load<float, N>(a.mul, sl, 0.f);
            float f[N];
#pragma unroll
            for (int i = 0; i < N; i++) f[i] = (float)v.v[i];
            uint32_t w[N / 4];
            codes_of<N, MUL>(f, mv.v, [&](int) -> const Coder& { return k; }, lim, w);
            __builtin_memcpy(o + sl.at, w, N);
        }
    }
}

// rows shorter than a vector, one per thread (100000 x 3 fp32 3.7 us)
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_rows_narrow(RqRowArgs a)
{
    const int C = (int)a.C, lim = (1 << (a.bits - 1)) - 1;
    for (int64_t m = blockIdx.x * (int64_t)256 + threadIdx.x; m < a.M; m += (int64_t)gridDim.x * 256) {
        const T* x = (const T*)a.x + m * a.x_ld;
        uint64_t big = 0;
        for (int c = 0; c < C; c++) {
            const uint64_t b = bits_of(a.mul ? (double)(float)x[c] * (double)a.mul[c] : (double)(float)x[c]);
            big = b > big ? b : big;
        }
        const float s = scale_of(big, a.bits, a.mode);
        const Coder k(s);
        a.scale[m] = s;
        if (!k.ok) set_status(a.status, ISEG_DEV_NONFINITE);
        for (int c = 0; c < C; c++) {
            const double v = a.mul ? (double)(float)x[c] * (double)a.mul[c] : (double)(float)x[c];
            a.codes[m * a.codes_ld + c] = k.ok ? (int8_t)code_wide(v, k, lim) : 0;
        }
    }
}

// ---------------------------------------------------------------------------
// columns
// ---------------------------------------------------------------------------
// Largest |v| (a double's bits) and sum of x of 64 columns over a strip of
// rows.  A block's threads take vectors of N columns: 64 / N of them side by
// side, the rows dealt to the others, four rows of each in flight.  4096 x 4096
// bf16 12.3 us (2.7 TB/s, a line of 128 bytes per row), with mul 14.4; k_cols_codes
// then finds x in the caches.
// A thread of the first 64 that holds a column gets its number, maximum and sum.
template <typename T, bool MUL>
__device__ __forceinline__ bool cols_part(const RqRowArgs& a, int64_t c0, int64_t m0, int64_t m1, int64_t& col,
                                          uint64_t& top, float& total)
{
    constexpr int N = RowVec<T>::N, G = 64 / N, RS = 256 / G;       // vectors across, rows at once
    __shared__ uint64_t rm[4][64];
    __shared__ float rs[4][64];
    const int tid = threadIdx.x, g = tid % G, r0 = tid / G, w = tid >> 6;
    const RowSlot<N> sl = row_slot<N>(c0 + g * N, a.C);
    float sum[N];
    uint64_t big[N];                          // exact magnitudes, formed where |fl(v)| reaches its largest so far
#pragma unroll
    for (int i = 0; i < N; i++) { sum[i] = 0.f; big[i] = 0; }
    uint32_t bt[N];
#pragma unroll
    for (int i = 0; i < N; i++) bt[i] = 0;
    for (int64_t m = m0 + r0; m < m1; m += RS * 4) {
        RowVec<T> xv[4];
        float mu[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {         // past the strip's end: the first row again, counted as nothing
            const int64_t mm = m + u * RS < m1 ? m + u * RS : m;
            xv[u] = slot_load<T, N>((const T*)a.x + mm * a.x_ld, sl);
            mu[u] = MUL ? a.mul[mm] : 1.f;
        }
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const bool in = m + u * RS < m1;
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float x = (float)xv[u].v[i];
                sum[i] += in ? x : 0.f;
                const uint32_t b = bits_of(MUL ? x * mu[u] : x);
                if (MUL) {
                    if (b >= bt[i]) {
                        const uint64_t e = bits_of((double)x * (double)mu[u]);
                        bt[i] = b;
                        big[i] = e > big[i] ? e : big[i];
                    }
                } else {
                    bt[i] = b > bt[i] ? b : bt[i];
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; i++)
        if (!MUL) big[i] = bits_of((double)__builtin_bit_cast(float, bt[i]));
    // over the rows of a wave: the lanes with the same g are G apart
#pragma unroll
    for (int o = G; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; i++) {
            const uint64_t t = __shfl_xor((unsigned long long)big[i], o, 64);
            big[i] = t > big[i] ? t : big[i];
            sum[i] += __shfl_xor(sum[i], o, 64);
        }
    if ((tid & 63) < G) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            rm[w][g * N + i] = big[i];
            rs[w][g * N + i] = sum[i];
        }
    }
    __syncthreads();
    if (tid >= 64) return false;
    // element tid of the vectors: column at + tid % N of its vector, unless it
    // repeats the vector before
    const RowSlot<N> mine = row_slot<N>(c0 + tid / N * N, a.C);
    if (tid % N < mine.dup) return false;
    col = mine.at + tid % N;
    top = rm[0][tid];
    total = rs[0][tid];
#pragma unroll
    for (int i = 1; i < 4; i++) {
        top = rm[i][tid] > top ? rm[i][tid] : top;
        total += rs[i][tid];
    }
    return true;
}

template <typename T, bool MUL>
__global__ __launch_bounds__(256) void k_cols_stats(RqRowArgs a, int64_t strip)
{
    const int64_t m0 = (int64_t)blockIdx.y * strip;
    const int64_t m1 = m0 + strip < a.M ? m0 + strip : a.M;
    int64_t c;
    uint64_t e;
    float s;
    if (!cols_part<T, MUL>(a, (int64_t)blockIdx.x * 64, m0, m1, c, e, s)) return;
    a.pmax[(int64_t)blockIdx.y * a.C + c] = e;
    a.psum[(int64_t)blockIdx.y * a.C + c] = s;
}

// the same for fewer columns than a vector: one thread per column and strip
template <typename T>
__global__ __launch_bounds__(64) void k_cols_stats_narrow(RqRowArgs a, int64_t strip)
{
    const int64_t m0 = (int64_t)blockIdx.y * strip;
    const int64_t m1 = m0 + strip < a.M ? m0 + strip : a.M;
    const int c = threadIdx.x;
    if (c >= a.C) return;
    uint64_t big = 0;
    float sum = 0.f;
    for (int64_t m = m0; m < m1; m++) {
        const float x = (float)((const T*)a.x)[m * a.x_ld + c];
        const uint64_t b = bits_of(a.mul ? (double)x * (double)a.mul[m] : (double)x);
        big = b > big ? b : big;
        sum += x;
    }
    a.pmax[(int64_t)blockIdx.y * a.C + c] = big;
    a.psum[(int64_t)blockIdx.y * a.C + c] = sum;
}

// largest magnitude and sum of a column from the strips' partials
__device__ __forceinline__ uint64_t col_join(const RqRowArgs& a, int64_t c, int strips, float* sum)
{
    uint64_t big = 0;
    float s = 0.f;
    for (int i0 = 0; i0 < strips; i0 += 8) {
        uint64_t b[8];
        float t[8];
#pragma unroll
        for (int u = 0; u < 8; u++) {         // past the end: the first of the eight again, counted as nothing
            const int64_t at = (int64_t)(i0 + u < strips ? i0 + u : i0) * a.C + c;
            b[u] = a.pmax[at];
            t[u] = a.psum[at];
        }
#pragma unroll
        for (int u = 0; u < 8; u++) {
            big = b[u] > big ? b[u] : big;
            s += i0 + u < strips ? t[u] : 0.f;
        }
    }
    *sum = s;
    return big;
}

// four words of four bytes each, turned: word x of the result holds byte x of
// every r[u]
__device__ __forceinline__ void turn4(const uint32_t* r, uint32_t* o)
{
    const uint32_t a0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400), a1 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602);
    const uint32_t b0 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400), b1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602);
    o[0] = (a0 & 0xffffu) | b0 << 16;
    o[1] = a0 >> 16 | (b0 & 0xffff0000u);
    o[2] = (a1 & 0xffffu) | b1 << 16;
    o[3] = a1 >> 16 | (b1 & 0xffff0000u);
}

// 16 codes of a column from words t[0 .. 3] to d; n (1 .. 16) of them exist
__device__ __forceinline__ void put16(const uint32_t* t, int8_t* d, int64_t n, bool wide)
{
    uint32_t v[4];
#pragma unroll
    for (int u = 0; u < 4; u++) v[u] = t[u];
    if (wide && n >= 16) {
        __builtin_memcpy(__builtin_assume_aligned(d, 16), v, 16);
    } else {
        const int e = n < 16 ? (int)n : 16;
        for (int u = 0; u < e; u++) d[u] = (int8_t)(t[u / 4] >> (u % 4 * 8));
    }
}

struct TurnArgs {
    const int8_t* in;
    int8_t* out;
    int64_t M, C, in_ld, out_ld;
    uint32_t tx, ty;             // blocks over the columns and over the rows
};

// Transposition of 128 x 128 codes: four rows of four columns per thread are
// turned by byte permutations into four words of four columns, so both sides
// move whole lines of 128 bytes.  4096 x 4096 7.5 us (4.5 TB/s).
// t: [column][rows / 4]; block (bx, by).
__device__ __forceinline__ void turn_codes(const TurnArgs& a, uint32_t (*t)[33], uint32_t bx, uint32_t by)
{
    const int64_t c0 = (int64_t)bx * 128;
    const bool wide = (a.out_ld & 15) == 0 && ((uintptr_t)a.out & 15) == 0;
    const int64_t mt = ceil_div64(a.M, 128);
    for (int64_t b = by; b < mt; b += a.ty) {
        const int64_t m0 = b * 128;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int e = threadIdx.x + i * 256, cq = e & 31, rq = e >> 5;     // columns / 4, rows / 4
            const int64_t c = c0 + cq * 4;
            uint32_t r[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int64_t m = m0 + rq * 4 + u < a.M ? m0 + rq * 4 + u : a.M - 1;
                const int8_t* p = a.in + m * a.in_ld + c;
                r[u] = 0;
                if (c + 4 <= a.C) {
                    __builtin_memcpy(&r[u], p, 4);
                } else {
                    for (int x = 0; x < 4; x++)
                        if (c + x < a.C) r[u] |= (uint32_t)(uint8_t)p[x] << (8 * x);
                }
            }
            uint32_t o[4];
            turn4(r, o);
#pragma unroll
            for (int x = 0; x < 4; x++) t[cq * 4 + x][rq] = o[x];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int e = threadIdx.x + i * 256, col = e >> 3, p = e & 7;
            const int64_t oc = c0 + col, m = m0 + p * 16;
            if (oc < a.C && m < a.M) put16(&t[col][p * 4], a.out + oc * a.out_ld + m, a.M - m, wide);
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void k_transpose_i8(TurnArgs a)
{
    __shared__ uint32_t t[128][33];
    turn_codes(a, t, blockIdx.x, blockIdx.y);
}

// Codes of 128 rows by 64 columns per step, turned by byte permutations and
// LDS: a thread codes one vector of N columns in each of four rows and leaves a
// word of four rows for each column (33 words apart, so a wave's columns fall
// on all the banks); rows of codes leave 16 bytes per lane, a whole line per
// column.  The block takes the scales from the strips' partials itself, or
// (strips = 0: at most 128 rows) from the columns, which spares a launch: 64 x
// 1024 bf16 8.1 us, 10.4 with k_cols_stats.  4096 x 4096 bf16 15 to 18 us: bound
// by the coding, 24 vector instructions per element (40 of 54 us at 16384 x 4096,
// by counters), with waits for the scales and each step's loads.  Blocks behind the cx * cy that code
// transpose the product's other operand (turn.ty = 0: none); of the linear
// layer's backward, 295 x 1024 x 2560 30.6 us, with a launch of its own 36.
template <typename T, bool MUL>
__global__ __launch_bounds__(256) void k_cols_codes(RqRowArgs a, int strips, uint32_t cx, uint32_t cy, TurnArgs turn)
{
    constexpr int N = RowVec<T>::N, G = 64 / N, RS = 256 / G;       // vectors across, row quads at once
    __shared__ uint32_t t[128][33];
    __shared__ float sc[64];
    const int tid = threadIdx.x, g = tid % G, rq0 = tid / G;
    if (blockIdx.x >= cx * cy) {
        const uint32_t b = blockIdx.x - cx * cy;
        turn_codes(turn, t, b % turn.tx, b / turn.tx);
        return;
    }
    const uint32_t bx = blockIdx.x % cx, by = blockIdx.x / cx;
    const int64_t c0 = (int64_t)bx * 64;
    const int lim = (1 << (a.bits - 1)) - 1;
    int64_t c = c0 + tid;
    uint64_t top = 0;
    float sum = 0.f;
    bool mine = tid < 64 && c < a.C;
    if (strips == 0) mine = cols_part<T, MUL>(a, c0, 0, a.M, c, top, sum);
    else if (mine) top = col_join(a, c, strips, &sum);
    if (mine) {
        const float s = scale_of(top, a.bits, a.mode);
        sc[c - c0] = s;
        if (by == 0) {
            a.scale[c] = s;
            if (a.sums) a.sums[c] = sum;
            if (!(s == s)) set_status(a.status, ISEG_DEV_NONFINITE);
        }
    }
    __syncthreads();
    const RowSlot<N> sl = row_slot<N>(c0 + g * N, a.C);
    Coder k[N];
#pragma unroll
    for (int i = 0; i < N; i++) k[i] = Coder(i >= sl.dup ? sc[sl.at - c0 + i] : 1.f);      // a repeated column's codes are dropped
    const bool wide = (a.codes_ld & 15) == 0 && ((uintptr_t)a.codes & 15) == 0;
    const int64_t mt = ceil_div64(a.M, 128);
    for (int64_t b = by; b < mt; b += cy) {
        const int64_t m0 = b * 128;
#pragma unroll
        for (int rq = rq0; rq < 32; rq += RS) {
            RowVec<T> xv[4];
            float mu[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int64_t m = m0 + rq * 4 + u < a.M ? m0 + rq * 4 + u : a.M - 1;
                xv[u] = slot_load<T, N>((const T*)a.x + m * a.x_ld, sl);
                mu[u] = MUL ? a.mul[m] : 1.f;
            }
            uint32_t w[4][N / 4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                float x[N], mm[N];
#pragma unroll
                for (int i = 0; i < N; i++) {
                    x[i] = (float)xv[u].v[i];
                    mm[i] = mu[u];
                }
                codes_of<N, MUL>(x, mm, [&](int i) -> const Coder& { return k[i]; }, lim, w[u]);
            }
#pragma unroll
            for (int q = 0; q < N / 4; q++) {
                const uint32_t r[4] = {w[0][q], w[1][q], w[2][q], w[3][q]};
                uint32_t o[4];
                turn4(r, o);
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (q * 4 + i >= sl.dup) t[sl.at - c0 + q * 4 + i][rq] = o[i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = tid; i < 64 * 8; i += 256) {
            const int col = i >> 3, p = i & 7;
            const int64_t oc = c0 + col, m = m0 + p * 16;
            if (oc < a.C && m < a.M) put16(&t[col][p * 4], a.codes + oc * a.codes_ld + m, a.M - m, wide);
        }
        __syncthreads();
    }
}

// the same for fewer columns than a vector, a code at a time
template <typename T>
__global__ __launch_bounds__(256) void k_cols_codes_narrow(RqRowArgs a, int strips)
{
    const int64_t c = blockIdx.x;
    const int lim = (1 << (a.bits - 1)) - 1;
    float sum;
    const float s = scale_of(col_join(a, c, strips, &sum), a.bits, a.mode);
    const Coder k(s);
    if (blockIdx.y == 0 && threadIdx.x == 0) {
        a.scale[c] = s;
        if (a.sums) a.sums[c] = sum;
        if (!k.ok) set_status(a.status, ISEG_DEV_NONFINITE);
    }
    for (int64_t m = (int64_t)blockIdx.y * 256 + threadIdx.x; m < a.M; m += (int64_t)gridDim.y * 256) {
        const float x = (float)((const T*)a.x)[m * a.x_ld + c];
        const double v = a.mul ? (double)x * (double)a.mul[m] : (double)x;
        a.codes[c * a.codes_ld + m] = k.ok ? (int8_t)code_wide(v, k, lim) : 0;
    }
}

constexpr int64_t kMaxCols = (int64_t)1 << 31;

// strips of rows whose partials a column's scale is taken from: blocks for the
// chip, at least 128 rows each
int64_t cols_strips(int64_t M, int64_t C)
{
    const int64_t tiles = ceil_div64(C, 64);
    int64_t n = ceil_div64(1024, tiles > 0 ? tiles : 1);
    const int64_t most = ceil_div64(M, 128);
    n = n < most ? n : most;
    return n > 0 ? (n < 256 ? n : 256) : 1;
}

template <typename T, bool MUL, int NW, int VPT>
int rows_grid(const RqRowArgs& a, hipStream_t s)
{
    constexpr int R = NW < 4 ? 4 / NW : 1;
    if (!slots_fit<T, NW, VPT>(a.C)) return ISEG_ERR_UNSUPPORTED;
    constexpr int threads = NW < 4 ? 256 : NW * 64;
    constexpr size_t lds = MUL ? (size_t)VPT * RowVec<T>::N * 4 * threads : 0;
    if (lds > 49152 && !lds_limit((const void*)k_quantize_rows<T, MUL, NW, VPT>, lds)) return ISEG_ERR_DEVICE;
    // with mul, what the chip holds at once: each block takes mul in
    const int64_t nb = ceil_div64(a.M, R), cap = MUL ? (NW < 4 ? 2048 : 256 * 32 / NW) : 4096;
    hipLaunchKernelGGL((k_quantize_rows<T, MUL, NW, VPT>), dim3((unsigned)(nb < cap ? nb : cap)), dim3(threads), lds, s, a);
    return launch_ok();
}

template <typename T, bool MUL>
int launch_rows_mul(const RqRowArgs& a, hipStream_t s)
{
    constexpr int N = RowVec<T>::N;
    const int64_t v = ceil_div64(a.C, N);
    if (a.C >= N) {
        if (v <= 64) return rows_grid<T, MUL, 1, 1>(a, s);
        if (v <= 128) return rows_grid<T, MUL, 1, 2>(a, s);
        if (v <= 256) return rows_grid<T, MUL, 4, 1>(a, s);
        if (v <= 512) return rows_grid<T, MUL, 4, 2>(a, s);
        if (v <= 1024) return rows_grid<T, MUL, 8, 2>(a, s);
        if (v <= 1536) return rows_grid<T, MUL, 8, 3>(a, s);
        if (v <= 2048) return rows_grid<T, MUL, 8, 4>(a, s);
        if (v <= 3 * 1024) return rows_grid<T, MUL, 16, 3>(a, s);
        if (v <= 4096) return rows_grid<T, MUL, 16, 4>(a, s);
        hipLaunchKernelGGL((k_quantize_rows_long<T, MUL>), dim3((unsigned)(a.M < kRowGridMax ? a.M : kRowGridMax)),
                           dim3(1024), 0, s, a);
        return launch_ok();
    }
    hipLaunchKernelGGL(k_quantize_rows_narrow<T>, dim3(grid_for(a.M, 256, 4096)), dim3(256), 0, s, a);
    return launch_ok();
}

template <typename T>
int launch_rows(const RqRowArgs& a, hipStream_t s)
{
    return a.mul ? launch_rows_mul<T, true>(a, s) : launch_rows_mul<T, false>(a, s);
}

int launch_turn(const TurnArgs& turn, hipStream_t s)
{
    if (turn.ty == 0) return ISEG_OK;
    hipLaunchKernelGGL(k_transpose_i8, dim3(turn.tx, turn.ty), dim3(256), 0, s, turn);
    return launch_ok();
}

template <typename T, bool MUL>
int launch_cols_mul(const RqRowArgs& a, const TurnArgs& turn, hipStream_t s)
{
    const unsigned ct = (unsigned)ceil_div64(a.C, 64);
    const int64_t strips = cols_strips(a.M, a.C);
    const int64_t strip = ceil_div64(a.M, strips);
    if (a.C < RowVec<T>::N) {
        hipLaunchKernelGGL(k_cols_stats_narrow<T>, dim3(1, (unsigned)strips), dim3(64), 0, s, a, strip);
        hipLaunchKernelGGL(k_cols_codes_narrow<T>, dim3((unsigned)a.C, grid_for(a.M, 256, 256)), dim3(256), 0, s, a,
                           (int)strips);
        return launch_turn(turn, s);
    }
    // one strip of a few rows: read again by the block that codes it
    const bool one = strips == 1 && a.M <= 128;
    if (!one) hipLaunchKernelGGL((k_cols_stats<T, MUL>), dim3(ct, (unsigned)strips), dim3(256), 0, s, a, strip);
    // blocks for the chip, each with the scales' work once
    const int64_t mt = ceil_div64(a.M, 128), most = ceil_div64(1024, ct);
    const int64_t gy = mt < most ? mt : most;
    const unsigned cy = (unsigned)(gy > 1 ? gy : 1);
    const int64_t blocks = (int64_t)ct * cy, extra = (int64_t)turn.tx * turn.ty;
    const bool both = blocks + extra < (int64_t)1 << 24;                // a launch's threads
    hipLaunchKernelGGL((k_cols_codes<T, MUL>), dim3((unsigned)(both ? blocks + extra : blocks)), dim3(256), 0, s, a,
                       one ? 0 : (int)strips, ct, cy, turn);
    return both ? launch_ok() : launch_turn(turn, s);
}

template <typename T>
int launch_cols(const RqRowArgs& a, const TurnArgs& turn, hipStream_t s)
{
    return a.mul ? launch_cols_mul<T, true>(a, turn, s) : launch_cols_mul<T, false>(a, turn, s);
}

TurnArgs turn_args(const TurnJob& j)
{
    const int64_t mt = ceil_div64(j.M, 128);
    return {j.in, j.out, j.M, j.C, j.in_ld, j.out_ld, (uint32_t)ceil_div64(j.C, 128), (uint32_t)(mt < 1024 ? mt : 1024)};
}

int rq_check(int32_t x_dtype, int32_t bits, int32_t mode)
{
    if (!is_float_dtype(x_dtype) || bits < 2 || bits > 8) return ISEG_ERR_ARG;
    if (mode != ISEG_SCALE_MAX && mode != ISEG_SCALE_POW2) return ISEG_ERR_ARG;
    return ISEG_OK;
}

}  // namespace

extern "C" int iseg_quantize_rows(const void* x, int32_t x_dtype, int64_t M, int64_t C, int64_t x_ld,
                                  const float* mul, int32_t bits, int32_t scale_mode, int8_t* codes,
                                  int64_t codes_ld, float* scale, int32_t* dev_status, hipStream_t stream)
{
    const int rc = rq_check(x_dtype, bits, scale_mode);
    if (rc != ISEG_OK) return rc;
    if (M < 0 || C < 0 || C >= kMaxCols || x_ld < C || codes_ld < C) return ISEG_ERR_SHAPE;
    if (M == 0) return ISEG_OK;
    if (!scale || (C > 0 && (!x || !codes))) return ISEG_ERR_ARG;
    RqRowArgs a = {};
    a.x = x; a.mul = mul; a.codes = codes; a.scale = scale;
    a.M = M; a.C = C; a.x_ld = x_ld; a.codes_ld = codes_ld; a.bits = bits; a.mode = scale_mode; a.status = dev_status;
    return x_dtype == ISEG_F32 ? launch_rows<float>(a, stream)
                               : x_dtype == ISEG_F16 ? launch_rows<f16_t>(a, stream) : launch_rows<bf16_t>(a, stream);
}

extern "C" size_t iseg_quantize_cols_ws(int64_t M, int64_t C)
{
    if (M < 0 || C < 0 || C > kMaxTurned) return 0;
    return ws_used((size_t)cols_strips(M, C) * (size_t)C * 12);
}

int quantize_cols_turn(const void* x, int32_t x_dtype, int64_t M, int64_t C, int64_t x_ld, const float* mul,
                       int32_t bits, int32_t scale_mode, int8_t* codes, int64_t codes_ld, float* scale, float* sums,
                       void* ws, size_t ws_bytes, int32_t* dev_status, const TurnJob* job, hipStream_t stream)
{
    const int rc = rq_check(x_dtype, bits, scale_mode);
    if (rc != ISEG_OK) return rc;
    if (M < 0 || C < 0 || C >= kMaxCols || x_ld < C || codes_ld < M) return ISEG_ERR_SHAPE;
    if (C > kMaxTurned || (job && job->C > kMaxTurned)) return ISEG_ERR_UNSUPPORTED;
    TurnArgs turn = {};
    if (job && job->M > 0 && job->C > 0) turn = turn_args(*job);
    if (C == 0) return launch_turn(turn, stream);
    if (!scale || (M > 0 && (!x || !codes))) return ISEG_ERR_ARG;
    if (!ws || ws_bytes < iseg_quantize_cols_ws(M, C)) return ISEG_ERR_WORKSPACE;
    RqRowArgs a = {};
    a.x = x; a.mul = mul; a.codes = codes; a.scale = scale; a.sums = sums;
    a.pmax = (uint64_t*)ws;
    a.psum = (float*)(a.pmax + cols_strips(M, C) * C);
    a.M = M; a.C = C; a.x_ld = x_ld; a.codes_ld = codes_ld; a.bits = bits; a.mode = scale_mode; a.status = dev_status;
    return x_dtype == ISEG_F32   ? launch_cols<float>(a, turn, stream)
           : x_dtype == ISEG_F16 ? launch_cols<f16_t>(a, turn, stream)
                                 : launch_cols<bf16_t>(a, turn, stream);
}

extern "C" int iseg_quantize_cols(const void* x, int32_t x_dtype, int64_t M, int64_t C, int64_t x_ld,
                                  const float* mul, int32_t bits, int32_t scale_mode, int8_t* codes,
                                  int64_t codes_ld, float* scale, float* sums, void* ws, size_t ws_bytes,
                                  int32_t* dev_status, hipStream_t stream)
{
    return quantize_cols_turn(x, x_dtype, M, C, x_ld, mul, bits, scale_mode, codes, codes_ld, scale, sums, ws, ws_bytes,
                              dev_status, nullptr, stream);
}

extern "C" int iseg_transpose_i8(const int8_t* in, int64_t M, int64_t C, int64_t in_ld, int8_t* out, int64_t out_ld,
                                 hipStream_t stream)
{
    if (M < 0 || C < 0 || C >= kMaxCols || in_ld < C || out_ld < M) return ISEG_ERR_SHAPE;
    if (C > kMaxTurned) return ISEG_ERR_UNSUPPORTED;
    if (M == 0 || C == 0) return ISEG_OK;
    if (!in || !out) return ISEG_ERR_ARG;
    return launch_turn(turn_args({in, M, C, in_ld, out, out_ld}), stream);
}
