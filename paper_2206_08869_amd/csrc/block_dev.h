// Device helpers that the training operators share: vectors of eight columns in three types, the 8-bit checkpoint's rounding,
// sums over the lanes of a row.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.h"

namespace iodf {

// Vectors at any element's address: rows of odd widths start anywhere, and this architecture loads and stores 16 bytes there too.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight elements as they lie in memory: what a load that is not waited for yet holds.
template <typename T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};

// From p on, of which the first n exist (n <= 0: none); the others are 0.
template <typename T>
__device__ __forceinline__ Raw8<T> fetch8(const T* p, int n) {
    Raw8<T> r;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const u32x4_any a = *(const u32x4_any*)((const char*)p + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[4 * i + j] = a[j];
        }
    } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : (T)0.f;
        __builtin_memcpy(r.w, t, sizeof(t));
    }
    return r;
}

__device__ __forceinline__ void widen8(const Raw8<float>& r, float v[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
}
__device__ __forceinline__ void widen8(const Raw8<__bf16>& r, float v[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen8(const Raw8<_Float16>& r, float v[8]) {
    _Float16 h[8];
    __builtin_memcpy(h, r.w, 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float v[8]) {
    widen8(fetch8(p, n), v);
}

// Rounded to nearest, ties to even.
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float v[8]) {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)v[i];
    if (n >= 8) {
        u32x4 w[sizeof(T) / 2];
        __builtin_memcpy(w, t, sizeof(t));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(u32x4_any*)(p + i * (8 / (sizeof(T) / 2))) = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = t[i];
    }
}

// ---- lanes ----

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// Sum over aligned runs of LPR lanes, the same in each of them.
template <int LPR>
__device__ __forceinline__ float lanes_sum(float v) {
    if (LPR >= 2) v += __uint_as_float(dpp<DPP_XOR1>(__float_as_uint(v)));
    if (LPR >= 4) v += __uint_as_float(dpp<DPP_XOR2>(__float_as_uint(v)));
    if (LPR >= 8) v += __uint_as_float(dpp<DPP_HALF_MIRROR>(__float_as_uint(v)));
    if (LPR >= 16) v += __uint_as_float(dpp<DPP_MIRROR>(__float_as_uint(v)));
    if (LPR >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if (LPR >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// N sums over the LPR threads of a row. Past a wave they meet in LDS, in two places by turns (`turn` counts the calls): with one barrier a
// call, nobody writes a place again before everybody has read it.
template <int LPR, int N>
struct RowSums {
    static constexpr int WAVES = LPR > 64 ? LPR / 64 : 1, W = WAVES <= 2 ? WAVES : WAVES <= 4 ? 4 : WAVES <= 8 ? 8 : 16;
    float at[2][N][W];
};
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float v[N], RowSums<LPR, N>& meet, int& turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<(LPR < 64 ? LPR : 64)>(v[k]);
    if (LPR > 64) {
        constexpr int W = RowSums<LPR, N>::W;
        float* const at = &meet.at[turn++ & 1][0][0];
        const int lane = threadIdx.x & 63;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) at[k * W + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
        // W lanes to a sum: one read, and the results in scalar registers
        const float mine = lanes_sum<W>(lane < N * W && lane % W < RowSums<LPR, N>::WAVES ? at[lane] : 0.f);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), k * W));
    }
}

// ---- checkpoint ----
// A group of 32 columns is four neighbouring lanes. Its exponent byte e is the biased exponent of its largest magnitude, one more if
// that magnitude would round to 128 steps; the step is 2^(e - 133), so that the magnitude is 64 to 127 of them. A power of two
// costs up to one of the eight bits against amax / 127, but a value is then exact in bfloat16 (seven bits and a sign) and goes
// to the matrix cores unrounded. e stays within 16..254: below, steps and their inverses would leave the normal numbers. 255
// stands for a group that holds a NaN or an infinity: all of it reads as NaN.
__device__ __forceinline__ float code_step(uint32_t e) {
    return e == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(((e > 6 ? e : 6) - 6) << 23);
}

// Codes of the eight values of this lane; the exponent byte is the same in the four lanes of the group.
__device__ __forceinline__ u32x2 encode8(const float v[8], uint32_t& e) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;  // as whole numbers, so that a NaN is the largest of all
        top = b > top ? b : top;
    }
    uint32_t o = dpp<DPP_XOR1>(top);
    top = o > top ? o : top;
    o = dpp<DPP_XOR2>(top);
    top = o > top ? o : top;
    const bool finite = top < 0x7f800000u;
    e = (top + 0x10000u) >> 23;
    e = e < 16 ? 16 : e > 254 ? 254 : e;
    const float inv = __uint_as_float((260 - e) << 23);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float r = fminf(fmaxf(rintf(v[i] * inv), -127.f), 127.f);
        w[i >> 2] |= ((uint32_t)(int)r & 0xffu) << (8 * (i & 3));
    }
    if (!finite) e = 255;
    return finite ? u32x2{w[0], w[1]} : u32x2{0, 0};
}

__device__ __forceinline__ void decode8(u32x2 q, float step, float v[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int)__builtin_amdgcn_sbfe((int)q[i >> 2], 8 * (i & 3), 8) * step;  // two instructions a value
}

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

// Rounded to bfloat16, two to a register.
__device__ __forceinline__ bf8 narrow8(const float v[8]) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    union { uint32_t w[4]; bf8 all; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf2 p = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
        u.w[i] = __builtin_bit_cast(uint32_t, p);
    }
    return u.all;
}

// One row's codes at columns c0.. (a multiple of 8) of a checkpoint with `pitch` columns.
__device__ __forceinline__ void store_codes(int8_t* q, uint8_t* e, long long row, int pitch, int c0, const float v[8]) {
    uint32_t ex;
    const u32x2 w = encode8(v, ex);  // every lane takes part: the group's maximum goes round its four lanes
    if (c0 < pitch) {
        *(u32x2*)(q + row * pitch + c0) = w;
        if ((c0 & 31) == 0) e[row * (pitch / 32) + c0 / 32] = (uint8_t)ex;
    }
}
// Eight codes and their exponent as they lie in memory (none past the pitch: zeros).
struct RawCodes {
    u32x2 q;
    uint32_t e;
};
__device__ __forceinline__ RawCodes fetch_codes(const int8_t* q, const uint8_t* e, long long row, int pitch, int c0) {
    RawCodes r = {u32x2{0, 0}, 16};
    if (c0 < pitch) {
        r.q = *(const u32x2*)(q + row * pitch + c0);
        r.e = e[row * (pitch / 32) + c0 / 32];
    }
    return r;
}
__device__ __forceinline__ void load_codes(const int8_t* q, const uint8_t* e, long long row, int pitch, int c0, float v[8]) {
    const RawCodes r = fetch_codes(q, e, row, pitch, c0);
    decode8(r.q, code_step(r.e), v);
}

// Makes the compiler forget what it has widened from these, so that it is widened again where it is used next and not held in four times the
// registers until then.
template <typename T>
__device__ __forceinline__ void forget(Raw8<T>& r) {
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) asm volatile("" : "+v"(r.w[i]));
}
__device__ __forceinline__ void forget(RawCodes& r) { asm volatile("" : "+v"(r.q), "+v"(r.e)); }

// ---- activations ----

// act(a), and its derivative. The logistic function is exp and a division: both ends are exact (exp overflows to infinity, 1 / inf = 0).
template <int ACT>
__device__ __forceinline__ float activate(float a, float& slope) {
    if (ACT == IODF_ACT_RELU) {
        slope = a > 0.f ? 1.f : 0.f;
        return a < 0.f ? 0.f : a;  // a NaN stays one
    }
    const float k = 1.5957691216057308f;  // 2 sqrt(2 / pi)
    const float arg = ACT == IODF_ACT_SILU ? a : k * (a + 0.044715f * a * a * a);
    const float s = 1.f / (1.f + __expf(-arg));
    const float bend = s * (1.f - s);
    if (ACT == IODF_ACT_SILU) slope = s + a * bend;
    else slope = bend == 0.f ? s : s + a * bend * k * (1.f + 0.134145f * a * a);  // far out a * a may be infinite
    return a * s;
}

}  // namespace iodf
