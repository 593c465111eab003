// coder.h -- scales and codes of the row and column quantizers.
//
// Every decision is exact although the work is float32.  With h = fl(x mul) (x
// itself without mul) and l = x mul - h (exact by one fma), |h| grows with
// |x mul|, so the largest exact magnitude is found among the elements with the
// largest |h|, and only those are formed in double (24 x 24 bits).  Magnitudes
// are compared as bit patterns, where a NaN or an infinity is larger than
// every finite value.  A code is n = floor(h / s + 1/2); where h / s + 1/2
// lies within 2^-14 of an integer (its error, of three roundings of at most
// 128, is below 2^-15), the sign of h - (n -+ 1/2) s + l settles it: (n + 1/2)
// s has 33 bits, its difference from h so near a half-step fits 24, and the
// last sum's sign is right however it rounds.
#pragma once

#include "rowops.h"

constexpr float kScaleMin = 1.17549435e-38f;      // 2^-126
constexpr uint64_t kAbs64 = 0x7fffffffffffffffull;
constexpr uint64_t kInf64 = 0x7ff0000000000000ull;

// scale of a largest magnitude given as a double's bits; NaN if there is none
__device__ __forceinline__ float scale_of(uint64_t big, int bits, int mode)
{
    if (big >= kInf64) return __builtin_nanf("");
    if (big == 0) return 1.f;
    const double t = __builtin_bit_cast(double, big);
    double s;
    if (mode == ISEG_SCALE_POW2) {
        int e;
        (void)frexp(t, &e);                        // t = f 2^e with f in [1/2, 1): 2^e is the power above t
        s = ldexp(1.0, e + 1 - bits);
    } else {
        s = t / (double)((1 << (bits - 1)) - 1);
    }
    const float f = (float)s;
    return f < kScaleMin ? kScaleMin : (f <= 3.4028234e38f ? f : __builtin_nanf(""));
}

__device__ __forceinline__ uint64_t bits_of(double v) { return __builtin_bit_cast(uint64_t, v) & kAbs64; }
__device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// How codes follow from a scale.  Outside [2^-60, 2^100], where a reciprocal,
// a product or its remainder may be subnormal or overflow, every code is
// formed in double.
struct Coder {
    float s, inv;
    bool ok, wide;
    __device__ __forceinline__ Coder() {}
    __device__ __forceinline__ explicit Coder(float s_)
        : s(s_), inv(1.f / s_), ok(s_ == s_), wide(!(s_ >= 8.6736174e-19f && s_ <= 1.2676506e30f))
    {
    }
};

// clamp(floor(v / s + 1/2), +-lim) of the exact v: an estimate within one,
// then the half-steps on either side of it
__device__ __forceinline__ int code_wide(double v, const Coder& k, int lim)
{
    const double sd = (double)k.s, q = fmin(fmax(v / sd, -128.0), 128.0);
    int n = (int)floor(q + 0.5);
    if (v - ((double)n + 0.5) * sd >= 0.0) n++;
    else if (v - ((double)n - 0.5) * sd < 0.0) n--;
    return n > lim ? lim : (n < -lim ? -lim : n);
}

// floor(h / s + 1/2) within one; `far` becomes the largest distance of h / s +
// 1/2 from a half-integer seen so far (kNear and above: near an integer)
__device__ __forceinline__ float code_fast(float h, const Coder& k, float& far)
{
    const float q = fmaf(h, k.inv, 0.5f), f = floorf(q);
    far = fmaxf(far, fabsf(q - f - 0.5f));
    return f;
}
constexpr float kNear = 0.5f - 6.1035156e-5f;

__device__ __forceinline__ float code_near(float n, float h, float l, const Coder& k)
{
    if (fmaf(-(n + 0.5f), k.s, h) + l >= 0.f) return n + 1.f;
    return fmaf(-(n - 0.5f), k.s, h) + l < 0.f ? n - 1.f : n;
}

__device__ __forceinline__ uint32_t pack4(const int* n)
{
    return (uint32_t)(uint8_t)n[0] | (uint32_t)(uint8_t)n[1] << 8 | (uint32_t)(uint8_t)n[2] << 16 | (uint32_t)n[3] << 24;
}

// codes of N values x (times m, exactly) as N bytes; coder(i) is element i's
template <int N, bool MUL, typename F>
__device__ __forceinline__ void codes_of(const float* x, const float* m, F coder, int lim, uint32_t* out)
{
    float f[N], far = 0.f;
    bool wide = false;
#pragma unroll
    for (int i = 0; i < N; i++) {
        f[i] = code_fast(MUL ? x[i] * m[i] : x[i], coder(i), far);
        wide |= coder(i).wide;
    }
    if (!(far < kNear)) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float h = MUL ? x[i] * m[i] : x[i];
            f[i] = code_near(f[i], h, MUL ? fmaf(x[i], m[i], -h) : 0.f, coder(i));
        }
    }
    int n[N];
    const float c = (float)lim;
#pragma unroll
    for (int i = 0; i < N; i++) n[i] = (int)fminf(fmaxf(f[i], -c), c);
    if (wide) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const Coder& k = coder(i);
            if (k.wide) n[i] = k.ok ? code_wide(MUL ? (double)x[i] * (double)m[i] : (double)x[i], k, lim) : 0;
        }
    }
#pragma unroll
    for (int i = 0; i < N / 4; i++) out[i] = pack4(n + 4 * i);
}
