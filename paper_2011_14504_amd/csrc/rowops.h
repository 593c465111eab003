// rowops.h -- device helpers of the row operators (layer norm, row and column
// quantizers, log probabilities): typed 16-byte vectors of rows that may start
// at any element, and float reductions over waves and blocks in a fixed order.
#pragma once

#include "iseg_common.h"

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

// N elements of a row, loaded and stored as one 16-byte access whatever the
// row's alignment (gfx950 takes global accesses at any byte address).
template <typename T>
struct RowVec {
    static constexpr int N = 16 / (int)sizeof(T);
    T v[N];
};

template <typename T>
__device__ __forceinline__ RowVec<T> row_load(const T* p)
{
    RowVec<T> r;
    __builtin_memcpy(&r, p, 16);
    return r;
}

// the first n (< N) elements; the others are `fill`
template <typename T>
__device__ __forceinline__ RowVec<T> row_load_part(const T* p, int n, T fill)
{
    RowVec<T> r;
#pragma unroll
    for (int i = 0; i < RowVec<T>::N; i++) r.v[i] = fill;
#pragma unroll
    for (int i = 0; i < RowVec<T>::N; i++)
        if (i < n) r.v[i] = p[i];
    return r;
}

template <typename T>
__device__ __forceinline__ void row_store(T* p, const RowVec<T>& r)
{
    __builtin_memcpy(p, &r, 16);
}

template <typename T>
__device__ __forceinline__ void row_store_part(T* p, const RowVec<T>& r, int n)
{
#pragma unroll
    for (int i = 0; i < RowVec<T>::N; i++)
        if (i < n) p[i] = r.v[i];
}

// One step of a wave reduction: the value of another lane by DPP, `old` where
// the pattern reads past its row (row_shr 1, 2, 4, 8, then the broadcasts of
// lanes 15 and 31 gather a wave's result in lane 63).
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float old, float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old),
                                                                 __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}

__device__ __forceinline__ float lane63_f32(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// sum over the 64 lanes, the same in every lane
__device__ __forceinline__ float wave_sum_f32(float v)
{
    v += dpp_f32<0x111>(0.f, v);
    v += dpp_f32<0x112>(0.f, v);
    v += dpp_f32<0x114>(0.f, v);
    v += dpp_f32<0x118>(0.f, v);
    v += dpp_f32<0x142>(0.f, v);
    v += dpp_f32<0x143>(0.f, v);
    return lane63_f32(v);
}

// largest of 64 lanes' unsigned values, the same in every lane
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_step(uint32_t v)
{
    const uint32_t t = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
    return t > v ? t : v;
}

__device__ __forceinline__ uint32_t wave_top_u32(uint32_t v)
{
    v = dpp_max_step<0x111>(v);
    v = dpp_max_step<0x112>(v);
    v = dpp_max_step<0x114>(v);
    v = dpp_max_step<0x118>(v);
    v = dpp_max_step<0x142>(v);
    v = dpp_max_step<0x143>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// sums of two values over the NW waves of a block, the same in every thread.
// red: 2 NW floats of LDS that no earlier call of this block may still read
// (callers alternate between two, or have a barrier between).
template <int NW>
__device__ __forceinline__ void block_sum2_f32(float& a, float& b, float* red)
{
    a = wave_sum_f32(a);
    b = wave_sum_f32(b);
    if (NW == 1) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (lane == 0) { red[2 * w] = a; red[2 * w + 1] = b; }
    __syncthreads();
    a = 0.f;
    b = 0.f;
#pragma unroll
    for (int i = 0; i < NW; i++) { a += red[2 * i]; b += red[2 * i + 1]; }
}

// A row of C >= N elements dealt to NT threads in vectors of N.  The row's last
// vector, when C is no multiple of N, starts N before the end instead: it
// repeats `dup` elements of the vector before it, which sums leave out and
// stores write a second time with the same bits.
template <int N>
struct RowSlot {
    int64_t at;      // first element
    int dup;         // repeated elements at its front; N if the thread has no vector here
};

template <int N>
__device__ __forceinline__ RowSlot<N> row_slot(int64_t c, int64_t C)
{
    if (c >= C) return {0, N};
    return c + N <= C ? RowSlot<N>{c, 0} : RowSlot<N>{C - N, (int)(c + N - C)};
}

template <typename T, int N>
__device__ __forceinline__ RowVec<T> slot_load(const T* row, const RowSlot<N>& s)
{
    RowVec<T> r;
    if (s.dup < N) {
        r = row_load(row + s.at);
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) r.v[i] = (T)0.f;
    }
    return r;
}

// N parameters of a column vector, `fill` without one
template <typename P, int N>
struct ParamVec {
    P v[N];
};

template <typename P, int N>
__device__ __forceinline__ ParamVec<P, N> param_load(const P* p, const RowSlot<N>& s, float fill)
{
    ParamVec<P, N> r;
    if (p && s.dup < N) {
        __builtin_memcpy(&r, p + s.at, sizeof(r));
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) r.v[i] = (P)fill;
    }
    return r;
}

// whether VPT vectors per thread of NW waves hold a row of C elements with only
// the last vector of a thread short (what the row kernels take for granted)
template <typename T, int NW, int VPT>
static inline bool slots_fit(int64_t C)
{
    const int64_t v = ceil_div64(C, RowVec<T>::N), nt = NW * 64;
    return C >= RowVec<T>::N && v > nt * (VPT - 1) && v <= nt * VPT;
}

// Workspace sizes: kNoWs of a call that touches none of it (one such buffer may
// then serve every stream), more than that of any other.
constexpr size_t kNoWs = 256;
static inline size_t ws_used(size_t bytes) { return bytes > 2 * kNoWs ? align256(bytes) : 2 * kNoWs; }

static inline bool is_float_dtype(int32_t t) { return t == ISEG_F32 || t == ISEG_F16 || t == ISEG_BF16; }

// whether no two rows of an output [T, H, D] with strides ld and hs overlap
static inline bool rows_apart(int64_t T, int64_t H, int64_t D, int64_t ld, int64_t hs)
{
    if (T < 1 || H < 1) return true;
    if (ld < 0 || hs < 0 || ld > (int64_t)1 << 40 || hs > (int64_t)1 << 40) return false;
    if (T > 1 && ld < D) return false;
    if (H > 1 && hs < D) return false;
    return T == 1 || H == 1 || ld >= (H - 1) * hs + D || hs >= (T - 1) * ld + D;
}

// launches walk their rows in a loop, so the grid may be cut at any count
constexpr int64_t kRowGridMax = 1 << 20;

// columns of a matrix that is quantized by column or transposed: a launch's threads
constexpr int64_t kMaxTurned = (int64_t)1 << 28;

// iseg_quantize_cols with, where `job` is given, the transposition of another
// matrix of codes (iseg_transpose_i8, its arguments checked by the caller) in
// the same launch.
struct TurnJob {
    const int8_t* in;
    int64_t M, C, in_ld;
    int8_t* out;
    int64_t out_ld;
};
int quantize_cols_turn(const void* x, int32_t x_dtype, int64_t M, int64_t C, int64_t x_ld, const float* mul,
                       int32_t bits, int32_t scale_mode, int8_t* codes, int64_t codes_ld, float* scale, float* sums,
                       void* ws, size_t ws_bytes, int32_t* dev_status, const TurnJob* job, hipStream_t stream);
